// Rows of a ragged batch go to the ends of their sequences in the paged cache, with more than a copy on the way: keys (and the
// queries of the same rows) rotated by their positions, or keys and values rounded to 4 bits, or both.  In a pair (a, b) of dims
// with the cosine c and sine s of the row's position and the pair's frequency:
//   a' = fl(a c) - fl(b s),   b' = fl(b c) + fl(a s);
// 4 bits: fp4.cuh.  Bound by memory: every row is read once and written once, a row of the table is read once per row and
// comes mostly from the caches.
//
// A thread has one unit of a row, two segments of S dims that a rotation by halves turns with one another: that unit of several heads
// of keys, queries and values in turn, then of its next row.  The cosines and sines stay in registers for a row.  Units lie next to
// each other in the lanes, then heads, then rows; a unit's segments lie half of the dims apart in any case, so that the lanes'
// segments make whole lines (one behind the other in a thread, 64 x 577 float32 took 158 us, now 100).
// A segment is 16 bytes, asked for up to kDepth units ahead into the thread's own places of a ring in shared memory (cp.async, no
// barriers), so that about 190 KB per SM are on their way.  On the way to 4 bits it is 32 bytes, a group of 16 dims in bf16 and half a
// group in float32, one unit ahead in registers (Shape).
#include "cache_rows.cuh"
#include "fp4.cuh"

namespace fz {
namespace {

constexpr int kThreads = 256;
constexpr int kBadShift = 16;   // a sample's counter: its CTAs that are done, and from this bit on those with a bad position
constexpr int kMostX = 2432;    // CTAs of a sample, at most
static_assert(kMostX < 1 << kBadShift, "a sample's CTAs are counted below the bad ones");

enum Pairs { kNone, kHalves, kAdjacent };

// Dims of a segment: 16 bytes, or 32 on the way to 4 bits, which saves more instructions than the half sectors of codes and scales cost
// (256 samples of 100 to 197 tokens of 6 x 64 bf16: 42 us with groups of two lanes, 33 of one; 300 of 100 to 300 of 4 x 64 float32: 62 with
// groups of four lanes, 47 of two, 54 of one, whose units fill the registers).  Those of 32 bytes are not asked for through the ring, whose
// copies would be written 16 bytes at a time, but one unit ahead in registers.  CTAs of an SM, and units of a thread's ring.
template <typename T, bool kFour, int P>
struct Shape {
    static constexpr int S = (kFour ? 32 : 16) / (int)sizeof(T), kChunks = S * (int)sizeof(T) / 16;   // 16 bytes of a segment
    static constexpr bool kRing = !kFour;
    static constexpr int kCtas = kFour && P != kNone ? 2 : 3;
    static constexpr int kDepth = kRing ? 8 : 2, kSmem = kRing ? kDepth * 2 * kThreads * 16 : 0;
};

// The next unit but one comes as far as the L2 meanwhile (1 x 32768 packed 103 us without it, 99 so; two units further 102).
__device__ __forceinline__ void to_l2(const void *a, const void *b) {
    asm volatile("prefetch.global.L2 [%0];" ::"l"(a));
    asm volatile("prefetch.global.L2 [%0];" ::"l"(b));
}
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// S dims, the even ones in e, the odd ones in o, two to a register pair.
template <int S> struct Segment {
    float2 e[S / 4], o[S / 4];
};
// 16 bytes as they lie in memory, at dim i of a segment.
template <int S> __device__ __forceinline__ void unpack(const uint4 &w, const float *, Segment<S> &x, int i) {
    x.e[i / 4] = make_float2(__uint_as_float(w.x), __uint_as_float(w.z));
    x.o[i / 4] = make_float2(__uint_as_float(w.y), __uint_as_float(w.w));
}
template <int S> __device__ __forceinline__ void unpack(const uint4 &w, const __nv_bfloat16 *, Segment<S> &x, int i) {
    auto low = [](uint32_t v) { return __uint_as_float(v << 16); };
    auto high = [](uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); };
    x.e[i / 4] = make_float2(low(w.x), low(w.y));
    x.o[i / 4] = make_float2(high(w.x), high(w.y));
    x.e[i / 4 + 1] = make_float2(low(w.z), low(w.w));
    x.o[i / 4 + 1] = make_float2(high(w.z), high(w.w));
}
template <int S> __device__ __forceinline__ void pack(const Segment<S> &x, int i, float *, uint4 &w) {
    w = make_uint4(__float_as_uint(x.e[i / 4].x), __float_as_uint(x.o[i / 4].x), __float_as_uint(x.e[i / 4].y), __float_as_uint(x.o[i / 4].y));
}
template <int S> __device__ __forceinline__ void pack(const Segment<S> &x, int i, __nv_bfloat16 *, uint4 &w) {
    auto both = [](float a, float b) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&p);
    };
    w = make_uint4(both(x.e[i / 4].x, x.o[i / 4].x), both(x.e[i / 4].y, x.o[i / 4].y), both(x.e[i / 4 + 1].x, x.o[i / 4 + 1].x),
                   both(x.e[i / 4 + 1].y, x.o[i / 4 + 1].y));
}

template <int S> struct CodesOf;   // the codes of a segment
template <> struct CodesOf<16> { using Type = unsigned long long; };
template <> struct CodesOf<8> { using Type = uint32_t; };

// Two segments of S dims, as they lie in memory.
template <typename T, int S>
struct Unit {
    static constexpr int kChunk = 16 / (int)sizeof(T), kChunks = S / kChunk;   // numbers of 16 bytes; 16 bytes of a segment
    uint4 w[2][kChunks];
    // From a thread's place in the ring, where its segments lie kThreads apart; and their copy to there.
    __device__ __forceinline__ void load(const uint4 *ring) {
        w[0][0] = ring[0];
        w[1][0] = ring[kThreads];
    }
    static __device__ __forceinline__ void ask(uint4 *ring, const T *a, const T *b, bool second) {
        cp_async16(ring, a);
        if (second) cp_async16(ring + kThreads, b);
    }
    // From memory: segments of 32 bytes, aligned to that or in two halves.
    __device__ __forceinline__ void load(const T *a, const T *b, bool aligned) {
#pragma unroll
        for (int i = 0; i + 1 < kChunks; i += 2) {
            load32(a + i * kChunk, w[0][i], w[0][i + 1], aligned);
            load32(b + i * kChunk, w[1][i], w[1][i + 1], aligned);
        }
    }
    static __device__ __forceinline__ void load32(const T *src, uint4 &x, uint4 &y, bool aligned) {
        if (aligned) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w), "=r"(y.x), "=r"(y.y), "=r"(y.z), "=r"(y.w)
                         : "l"(src));
        } else {
            x = reinterpret_cast<const uint4 *>(src)[0];
            y = reinterpret_cast<const uint4 *>(src)[1];
        }
    }
    __device__ __forceinline__ void store(T *a, T *b, bool second) const {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            reinterpret_cast<uint4 *>(a)[i] = w[0][i];
            if (second) reinterpret_cast<uint4 *>(b)[i] = w[1][i];
        }
    }
    __device__ __forceinline__ void get(int s, Segment<S> &x) const {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) unpack<S>(w[s][i], (const T *)nullptr, x, i * kChunk);
    }
    __device__ __forceinline__ void set(int s, const Segment<S> &x) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) pack<S>(x, i * kChunk, (T *)nullptr, w[s][i]);
    }
};

// N floats, 16- or 8-byte aligned.
template <int N> __device__ __forceinline__ void load_floats(const float *src, float *x) {
    if constexpr (N == 2) {
        const float2 v = *reinterpret_cast<const float2 *>(src);
        x[0] = v.x, x[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(src + i);
            x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
        }
    }
}
// Every product is rounded by itself: the sums go one by one, since the assembler makes mul2 and add2 one operation with one rounding.
__device__ __forceinline__ void turn(float2 &a, float2 &b, float2 c, float2 s) {
    const float2 ac = mul2(a, c), bs = mul2(b, s), bc = mul2(b, c), as = mul2(a, s);
    a = make_float2(__fadd_rn(ac.x, -bs.x), __fadd_rn(ac.y, -bs.y));
    b = make_float2(__fadd_rn(bc.x, as.x), __fadd_rn(bc.y, as.y));
}
// Cosines and sines of a unit's S pairs: those of the first segment's dims with the second's (even ones, odd ones), or of
// neighbours, that is of an even dim with the next, in each.
template <int S, int P>
struct Angles {
    float2 c[S / 2], s[S / 2];
    __device__ __forceinline__ void load(const float *row, int half, int a, int b, bool first, bool second) {
        float x[S], y[S];
        if constexpr (P == kHalves) {
            load_floats<S>(row + a, x);
            load_floats<S>(row + half + a, y);
#pragma unroll
            for (int i = 0; i < S / 4; ++i) {
                c[i] = make_float2(x[4 * i], x[4 * i + 2]), c[S / 4 + i] = make_float2(x[4 * i + 1], x[4 * i + 3]);
                s[i] = make_float2(y[4 * i], y[4 * i + 2]), s[S / 4 + i] = make_float2(y[4 * i + 1], y[4 * i + 3]);
            }
        } else {
            if (first) {
                load_floats<S / 2>(row + a / 2, x);
                load_floats<S / 2>(row + half + a / 2, y);
            }
            if (second) {
                load_floats<S / 2>(row + b / 2, x + S / 2);
                load_floats<S / 2>(row + half + b / 2, y + S / 2);
            }
#pragma unroll
            for (int i = 0; i < S / 2; ++i) {
                c[i] = make_float2(x[2 * i], x[2 * i + 1]);
                s[i] = make_float2(y[2 * i], y[2 * i + 1]);
            }
        }
    }
    __device__ __forceinline__ void turn_unit(Segment<S> &a, Segment<S> &b, bool first, bool second) const {
        if constexpr (P == kHalves) {
#pragma unroll
            for (int i = 0; i < S / 4; ++i) {
                turn(a.e[i], b.e[i], c[i], s[i]);
                turn(a.o[i], b.o[i], c[S / 4 + i], s[S / 4 + i]);
            }
        } else {
            if (first) {
#pragma unroll
                for (int i = 0; i < S / 4; ++i) turn(a.e[i], a.o[i], c[i], s[i]);
            }
            if (second) {
#pragma unroll
                for (int i = 0; i < S / 4; ++i) turn(b.e[i], b.o[i], c[S / 4 + i], s[S / 4 + i]);
            }
        }
    }
};

// Rows of CTAs as in k_cache_append: one per sample, and one more for the lengths while the grid has room for it.  `lanes`:
// threads that share the heads of a unit.
template <typename T, bool kFour, int P>
__global__ void __launch_bounds__(kThreads, Shape<T, kFour, P>::kCtas) k_cache_store(CacheStoreParams p, int units, int lanes) {
    using X = Shape<T, kFour, P>;
    constexpr int S = X::S, kDepth = X::kDepth, kSlot = 2 * kThreads, kShare = 16 / S;   // kShare: lanes of a group of 16 dims
    extern __shared__ __align__(16) uint4 ring[];   // [kDepth][2][kThreads]
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

    // this thread's unit: its dims, whether they are rotated, and its first head and row
    const int per_row = units * lanes, side = kThreads / per_row, mine = tid / per_row, u = tid % units, lane = tid / units % lanes;
    // where values (and keys and queries but for a rotation by halves) have its segments, and where keys and queries have them
    const int plain_a = S * u, plain_b = S * (u + units);
    const int turning = P == kHalves ? p.turned / (2 * S) : 0;   // units that a rotation by halves turns, the first ones
    const int a = P == kHalves && u >= turning ? p.turned + S * (u - turning) : plain_a;
    const int b = P != kHalves ? plain_b : u < turning ? a + p.turned / 2 : a + S * (units - turning);
    const bool turn_a = P == kHalves ? u < turning : P == kAdjacent && a < p.turned, turn_b = P == kHalves ? turn_a : P == kAdjacent && b < p.turned;
    const bool second = b < c.dim, plain_second = plain_b < c.dim;   // (where S divides the dims an odd number of times)
    const int heads = p.q ? p.heads : 0;
    const int r_first = mine < side && rows_ok ? (int)blockIdx.x * side + mine : n, r_step = (int)gridDim.x * side;
    // the next unit to ask for: keys, queries and values of a row (kinds 0, 1, 2), a thread's heads in turn; its place in the ring
    int ask_r = r_first, ask_kind = 0, ask_left = 0, ask_at = 0;
    const T *ask_a = nullptr, *ask_b = nullptr;
    bool ask_second = false;
    auto find = [&]() {   // the first head of this thread from (ask_r, ask_kind) on
        for (;;) {
            if (ask_kind == 3) {
                ask_kind = 0;
                ask_r += r_step;
            }
            ask_left = (ask_kind == 1 ? heads : c.kv_heads) - lane;
            if (ask_r >= n || ask_left > 0) break;
            ++ask_kind;
        }
        const unsigned char *base = ask_kind == 0 ? p.k : ask_kind == 1 ? p.q : p.v;
        const long long stride = ask_kind == 0 ? p.k_stride : ask_kind == 1 ? p.q_stride : p.v_stride;
        const T *src = reinterpret_cast<const T *>(base + (size_t)(o0 + ask_r) * stride) + (size_t)lane * c.dim;
        ask_a = src + (ask_kind == 2 ? plain_a : a);
        ask_b = src + (ask_kind == 2 ? plain_b : b);
        ask_second = ask_kind == 2 ? plain_second : second;
    };
    find();
    const int ask_step = lanes * c.dim;
    const bool aligned = ((reinterpret_cast<uintptr_t>(p.k) | reinterpret_cast<uintptr_t>(p.v) | reinterpret_cast<uintptr_t>(p.q) | (uintptr_t)p.k_stride |
                           (uintptr_t)p.v_stride | (uintptr_t)p.q_stride) & 31u) == 0;
    Unit<T, S> ahead;
    auto ask = [&]() {
        if (ask_r < n) {
            if constexpr (X::kRing) Unit<T, S>::ask(ring + ask_at * kSlot + tid, ask_a, ask_b, ask_second);
            else ahead.load(ask_a, ask_b, aligned);
            ask_a += ask_step;
            ask_b += ask_step;
            ask_left -= lanes;
            if constexpr (!X::kRing)
                if (ask_left > 0) to_l2(ask_a, ask_b);
            if (ask_left <= 0) {
                ++ask_kind;
                find();
            }
        }
        if constexpr (X::kRing) {
            cp_async_commit();
            ask_at = ask_at + 1 == kDepth ? 0 : ask_at + 1;
        }
    };
#pragma unroll 1
    for (int d = 0; d < kDepth - 1; ++d) ask();

    int bad = !rows_ok ? FUSION_DEV_BAD_OFFSETS : at < 0 || at > c.capacity || n > c.capacity - at ? FUSION_DEV_BAD_CACHE : 0;
    const unsigned *pages = reinterpret_cast<const unsigned *>(c.table) + (size_t)slot * c.max_pages;
    // page and position of a row, read a row ahead (0 and 0 behind the last), and its angles, asked for behind the last use of those
    // of the row before
    auto page_of = [&](int r) { return r < n ? pages[(at + r) >> c.shift] : 0u; };
    auto position_of = [&](int r) { return P == kNone ? 0u : r >= n ? 0u : (unsigned)(p.positions ? p.positions[o0 + r] : at + r); };
    auto known_of = [&](unsigned pos) { return P == kNone || pos < (unsigned)p.table_rows; };   // a row without a position in the table is left out
    Angles<S, P> w;
    const bool turned = turn_a || turn_b;
    auto load_angles = [&](int r, unsigned pos) {
        if constexpr (P != kNone)
            if (turned && r < n && known_of(pos)) w.load(p.table + (size_t)pos * p.turned, p.turned / 2, a, b, turn_a, turn_b);
    };
    bool wrong = false;
    unsigned page = 0u, pos = 0u;
    if (!bad) {
        page = page_of(r_first);
        pos = position_of(r_first);
        for (int e = (at >> c.shift) + tid; n > 0 && e <= (at + n - 1) >> c.shift; e += kThreads) wrong |= pages[e] >= c.num_pages;
        load_angles(r_first, pos);
    }
    if (named_twice<kThreads>(p.in, B, i, slot)) bad |= FUSION_DEV_BAD_IDS;
    if (__syncthreads_or(wrong)) bad |= FUSION_DEV_BAD_CACHE;
    if (bad) {   // nothing of this sample is written, and its slot's length stays (also where it is named twice)
        if (blockIdx.x == 0 && tid == 0) {
            raise_status(p.status, bad);
            if (!p.in_place) p.lengths_out[slot] = at;
        }
        cp_async_wait<0>();
        return;
    }
    const unsigned low = (1u << c.shift) - 1u;
    bool bad_position = false;
    int have_at = 0;
    for (int r = r_first; r < n; r += r_step) {
        const unsigned place = (unsigned)(at + r) & low;
        const bool known = known_of(pos);
        bad_position |= !known;
        const unsigned next_page = page_of(r + r_step), next_pos = position_of(r + r_step);
        const size_t row = (size_t)(o0 + r), first_row = (size_t)((page * (unsigned)c.kv_heads) << c.shift) + place;   // of key head 0 in the pools
        auto next_unit = [&](Unit<T, S> &v) {
            if constexpr (X::kRing) {
                ask();
                cp_async_wait<kDepth - 1>();
                v.load(ring + have_at * kSlot + tid);
                have_at = have_at + 1 == kDepth ? 0 : have_at + 1;
            } else {
                v = ahead;
                ask();
            }
        };
        auto turn_in_place = [&](Unit<T, S> &v) {
            if constexpr (P != kNone)
                if (turned) {
                    Segment<S> xa, xb;
                    v.get(0, xa);
                    v.get(1, xb);
                    w.turn_unit(xa, xb, turn_a, turn_b);
                    if (turn_a) v.set(0, xa);
                    if (turn_b) v.set(1, xb);
                }
        };
        // keys or values, from this thread's first head on
        auto to_pool = [&](unsigned char *pool, unsigned char *scales, int da, int db, bool two, bool turns) {
            const size_t row0 = first_row + ((size_t)lane << c.shift), step = (size_t)lanes << c.shift;
            if constexpr (kFour) {
                using Codes = typename CodesOf<S>::Type;
                const unsigned mask = kShare == 1 ? 0u : ((1u << kShare) - 1u) << (tid & 31 & ~(kShare - 1));
                unsigned char *codes = pool + row0 * (c.dim / 2) + da / 2, *z = scales + row0 * p.s.bytes;
                const int apart = (db - da) / 2, za = da / 16, zb = db / 16;
#pragma unroll 1
                for (int h = lane; h < c.kv_heads; h += lanes, codes += step * (c.dim / 2), z += step * p.s.bytes) {
                    Unit<T, S> v;
                    next_unit(v);
                    if (!known) continue;
                    Segment<S> xa, xb;
                    v.get(0, xa);
                    v.get(1, xb);
                    if constexpr (P != kNone)
                        if (turns) w.turn_unit(xa, xb, turn_a, turn_b);
                    uint32_t sa, sb;
                    const Codes ca = (Codes)quantise<S>(xa.e, xa.o, mask, sa), cb = (Codes)quantise<S>(xb.e, xb.o, mask, sb);
                    *reinterpret_cast<Codes *>(codes) = ca;
                    *reinterpret_cast<Codes *>(codes + apart) = cb;
                    if (u % kShare == 0) {
                        z[za] = (unsigned char)sa;
                        z[zb] = (unsigned char)sb;
                    }
                    if (u == 0)   // (the bytes behind the last scale)
                        for (int x = c.dim / 16; x < p.s.bytes; ++x) z[x] = 0;
                }
            } else {
                T *dst = reinterpret_cast<T *>(pool) + row0 * c.dim + da;
#pragma unroll 1
                for (int h = lane; h < c.kv_heads; h += lanes, dst += step * c.dim) {
                    Unit<T, S> v;
                    next_unit(v);
                    if (!known) continue;
                    if (turns) turn_in_place(v);
                    v.store(dst, dst + (db - da), two);
                }
            }
        };
        to_pool(c.k, p.s.k, a, b, second, turned);
#pragma unroll 1
        for (int h = lane; P != kNone && h < heads; h += lanes) {
            Unit<T, S> v;
            next_unit(v);
            if (!known) continue;
            turn_in_place(v);
            T *dst = reinterpret_cast<T *>(p.q_out) + (row * heads + h) * c.dim;
            v.store(dst + a, dst + b, second);
        }
        load_angles(r + r_step, next_pos);
        to_pool(c.v, p.s.v, plain_a, plain_b, plain_second, false);
        if (u == 0 && lane == 0 && known) {
            const size_t s = ((size_t)page << c.shift) + place;
            if (c.sizes) c.sizes[s] = p.sizes ? p.sizes[row] : 1.0f;
            if (c.weights) c.weights[s] = p.scores ? p.scores[row] : 0.0f;
        }
        page = next_page;
        pos = next_pos;
    }
    cp_async_wait<0>();
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

// Units of a row that a thread has, if `lanes` threads share a unit's heads.
int units_of(int lanes, int kv_heads, int heads) { return 2 * ceil_div(kv_heads, lanes) + ceil_div(heads, lanes); }
// Units of a row that a thread has at most, where it can choose, and has at least in all of its CTA's rows, where there is work
// enough: a CTA starts with four loads that wait for one another.  (At most 8 of a row and 16 in all: 1 x 32768 packed 115 us, now 103;
// 32 in all 119, since the last CTAs then leave SMs idle.  64 x 577 float32 100, now 96; 256 samples of 100 to 197 41, now 39.)  Half as
// many of a row where the CTAs would not fill the GPU one and a half times (10 samples of 47 of 16 + 16 + 64 heads of 128 float32 20.6
// us, now 13; 195 of 249 of 8 + 8 + 16 heads of 32 63, now 56).
constexpr int kUnits = 24;
// How many threads share a unit's heads: of the numbers that let no more rows lie side by side than there are, one that leaves the
// fewest threads idle; of those the smallest, since a thread reads the angles of its unit once per row.
int lanes_of(int units, int kv_heads, int heads, long long rows, long long batch, int places) {
    const int more = heads > kv_heads ? heads : kv_heads, most = more < kThreads / units ? more : kThreads / units;
    int best = most;
    double best_used = 0.0;
    for (int lanes = most; lanes >= 1; --lanes) {
        const int side = kThreads / (units * lanes), mine = units_of(lanes, kv_heads, heads);
        if (side > rows && lanes < most) break;
        const double used = (double)side * units * (2 * kv_heads + heads) / mine;
        const int at_most = (rows + side - 1) / side * batch * 2 >= 3 * places ? kUnits : kUnits / 2;
        if (used > best_used * 1.02 || (used >= best_used * 0.999 && mine <= at_most)) {
            best = lanes;
            best_used = used;
        }
    }
    return best;
}

template <typename T, bool kFour, int P>
cudaError_t launch(const CacheStoreParams &p, cudaStream_t s) {
    using X = Shape<T, kFour, P>;
    constexpr int S = X::S;
    int places = 0;
    const cudaError_t e = resident_ctas<k_cache_store<T, kFour, P>, kThreads>(X::kSmem, places);
    if (e != cudaSuccess) return e;
    const int heads = p.q ? p.heads : 0;
    // in segments of 16 bytes an even number, if there is room for it, so that the lanes' segments end where sectors do (11 samples of 556
    // of 16 + 16 + 64 heads of 80 bf16 51.8 us, now 39.4)
    int units = ceil_div(p.c.dim, 2 * S);
    if (!kFour && units % 2 && S * (units + 1) <= p.c.dim - (P == kHalves ? p.turned / 2 : 0)) ++units;
    // (samples of more rows than the cache has room for, or than there are, write nothing)
    long long most = p.in.max_tokens < p.c.capacity ? p.in.max_tokens : p.c.capacity;
    if (most > p.in.max_rows) most = p.in.max_rows;
    if (most < 1) most = 1;
    const int lanes = lanes_of(units, p.c.kv_heads, heads, most, p.in.max_batch, places), side = kThreads / (units * lanes);
    // as many rows a CTA as make its start worth while, unless that leaves SMs without two rounds of CTAs
    const long long steps = (most + side - 1) / side, per_step = units_of(lanes, p.c.kv_heads, heads);
    long long turns = (kUnits + per_step - 1) / per_step;
    const long long least = (2ll * places + p.in.max_batch) / (p.in.max_batch + 1);   // CTAs of a sample
    if (turns > steps / least) turns = steps / least;
    if (turns < 1) turns = 1;
    long long x = (steps + turns - 1) / turns;
    if (x > kMostX) x = kMostX;
    static_assert(FUSION_CACHE_MAX_BATCH <= kMostY, "a row of CTAs per sample");
    const dim3 grid((unsigned)x, (unsigned)(p.in.max_batch < kMostY ? p.in.max_batch + 1 : kMostY));
    return launch_after(k_cache_store<T, kFour, P>, grid, kThreads, X::kSmem, 1, s, p, units, lanes);
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
