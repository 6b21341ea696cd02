// What the kernels of the paged key-value cache share: the cache as the device sees it, the scratch they
// carve from the caller's workspace, and the host's launchers.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

#include "common.cuh"

namespace fz {

// Row of token `place` of page `page` for key head h in the pools: (page * kv_heads + h) * page_tokens + place,
// an unsigned 32-bit number (the host refuses pools of more rows); its bytes are rows * dim * element size apart.
struct Cache {
    int max_batch, max_pages, shift, kv_heads, dim;   // shift: log2 of page_tokens
    unsigned num_pages;
    int capacity;                   // max_pages * page_tokens
    unsigned char *k, *v;
    float *sizes, *weights;         // by slot: page * page_tokens + place; NULL: none
    const int *table;
    const int *lengths;
};

// An entry of the page table or a length; kEarly: past the L1 cache (wait_for_previous).
template <bool kEarly> __device__ __forceinline__ int cache_entry(const int *p) { return kEarly ? __ldcg(p) : *p; }
// The page that holds position pos of sequence b; false when its id is out of range.
template <bool kEarly = false>
__device__ __forceinline__ bool cache_page(const Cache &c, int b, int pos, unsigned &page) {
    page = (unsigned)cache_entry<kEarly>(&c.table[(size_t)b * c.max_pages + (pos >> c.shift)]);
    return page < c.num_pages;
}
// Length of sequence b, or -1 when it is out of range.
template <bool kEarly = false>
__device__ __forceinline__ int cache_length(const Cache &c, int b) {
    const int n = cache_entry<kEarly>(&c.lengths[b]);
    return n >= 0 && n <= c.capacity ? n : -1;
}

// Every kernel of the cache calls is a programmatic dependent of the one before it on the stream: it is launched while that one
// still runs, and waits for its end (and its writes) before it touches memory that a kernel may have written.  All of a kernel's
// CTAs wait, also those without work, so that its end implies the end of the ones before it.  k_cache_weights alone reads something
// before its wait, lengths and pages: it starts when the attention kernel's CTAs have all waited, so the kernels that wrote those
// have ended and their writes are in the L2 cache, but only the wait would make an SM forget older lines in its L1: it reads them
// past the L1 (the attention kernel does not, whose pages' other entries the L1 keeps: 16 x 577 float32 19.4 us, past it 20.9).
__device__ __forceinline__ void wait_for_previous() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename... P, typename... A>
inline cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute a[2];
    a[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a[0].val.programmaticStreamSerializationAllowed = 1;
    a[1].id = cudaLaunchAttributeClusterDimension;
    a[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = a;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// Host: as many CTAs of a kernel as the GPU holds at once, and its `smem` bytes of dynamic shared memory allowed.  What depends on the
// kernel and the device alone is asked once (asking costs the host 4 us a call).
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

// Query heads times places of a cache, at most (the host refuses more).
constexpr long long kCacheMaxHeadTokens = 1ll << 36;

// Scratch behind the counters of the workspace.  Attention: log-sum-exps, partial results of sequences that
// several CTAs share, logits (only where weights are accumulated).  Eviction: the kept slots and their counts.
constexpr int kCacheMaxCtas = 2048;   // CTAs of the attention kernel; each has two partial results at most
constexpr int kCacheMaxWide = 512;    // those of four warps
constexpr int kCacheMaxQ = 16;       // query heads of a key head that one CTA takes, at most
struct CacheWs {
    size_t counters, lse, part_ml, part, logits, keep, plan, total;
    long long lstride;               // logits of one (sequence, head)
};
inline CacheWs cache_ws_layout(int max_batch, int max_pages, int page_tokens, int kv_heads, int dim, int heads, bool weights) {
    const size_t b = max_batch > 0 ? max_batch : 1, cap = (size_t)max_pages * page_tokens;
    const int group = heads / kv_heads, nq = group <= 8 ? 8 : kCacheMaxQ;
    CacheWs L;
    L.lstride = (long long)((cap + 3) / 4 * 4);
    const size_t ctas = dim <= 128 ? kCacheMaxCtas : kCacheMaxWide;
    L.counters = 0;
    L.lse = align256(sizeof(int) * (size_t)kWsCounters);
    L.part_ml = L.lse + align256(b * heads * 4);
    L.part = L.part_ml + align256(2 * ctas * nq * 8);
    L.logits = L.part + align256(2 * ctas * nq * dim * 4);
    const size_t attn = L.logits + (weights ? align256(b * heads * (size_t)L.lstride * 4) : 0);
    L.plan = L.lse;
    L.keep = L.plan + align256(b * 8);
    const size_t evict = weights ? L.keep + align256(b * cap * 4) : 0;
    L.total = attn > evict ? attn : evict;
    return L;
}

struct CacheAttnParams {
    Cache c;
    const void *q;
    long long q_stride;    // elements between the sequences' queries
    int heads, group;      // group: query heads of a key head
    float scale2;          // scale * log2(e)
    int window, sinks;     // set_visible; window 0: every token is visible
    int most;              // visible tokens of a sequence, at most
    void *out;
    float *lse;            // [max_batch, heads] base 2
    float2 *part_ml;       // (maximum, sum) of the partial results' rows
    float *part;
    float *logits;         // base 2; NULL: no weights
    long long lstride;
    int *counters;
    int *status;
};
// The caller's window and sinks (any numbers from 0) over p.c.capacity positions.  A window over all of them is none, and sinks
// beyond the positions that a window leaves say nothing more, so their sum is at most the capacity (2^30) and cannot overflow.
inline void set_visible(CacheAttnParams &p, int window, int sinks) {
    const int capacity = p.c.capacity;
    p.window = window < capacity ? window : 0;
    p.sinks = sinks < capacity - p.window ? sinks : capacity - p.window;
    p.most = p.window ? p.window + p.sinks : capacity;
}
// Visible tokens of a sequence of n tokens: the j-th is position j (j < sinks) or j + n - visible.
__host__ __device__ __forceinline__ int visible(const CacheAttnParams &p, int n) {
    return p.window ? min(n, p.window + p.sinks) : n;
}
cudaError_t launch_cache_attention_bf16(const CacheAttnParams &p, cudaStream_t s);   // without the weights
cudaError_t launch_cache_attention(int dtype, const CacheAttnParams &p, cudaStream_t s);
cudaError_t launch_cache_weights(const CacheAttnParams &p, cudaStream_t s);           // after the attention

// The scales of a cache in 4 bits: `bytes` of a row, a multiple of 4.
struct PackedScales {
    unsigned char *k, *v;
    int bytes;
};
struct PackedAttnParams : CacheAttnParams {
    PackedScales s;
};
cudaError_t launch_packed_attention(int dtype, const PackedAttnParams &p, cudaStream_t s);

struct CacheAppendParams {
    Cache c;
    Ragged in;
    const unsigned char *k, *v;
    long long k_stride, v_stride;   // bytes between rows
    const float *sizes, *scores;
    int *lengths_out;
    int in_place;                   // lengths_out is the cache's own
    int *counters;
    int *status;
};
cudaError_t launch_cache_append(int dtype, const CacheAppendParams &p, cudaStream_t s);

// Keys and queries rotated on the way (turned > 0), or a cache in 4 bits (s.k), or both.
struct CacheStoreParams : CacheAppendParams {
    PackedScales s;
    const float *table;
    int table_rows, turned;         // turned: dims that are rotated
    const int *positions;
    const unsigned char *q;         // NULL: none
    long long q_stride;             // bytes between rows
    int heads;
    unsigned char *q_out;
};
cudaError_t launch_cache_store(int dtype, int pairs, const CacheStoreParams &p, cudaStream_t s);

struct CacheReadParams {
    Cache c;
    PackedScales s;                      // s.k NULL: not in 4 bits
    Ragged in;
    const int *starts;
    unsigned char *k_out, *v_out;
    float *sizes_out, *weights_out;
    int *status;
};
cudaError_t launch_cache_read(int dtype, const CacheReadParams &p, cudaStream_t s);

struct CacheEvictParams {
    Cache c;
    const int *budget;
    int sinks, recent;
    const int *table_out;
    int pages_out;                  // entries of a row of table_out
    int in_place;                   // table_out is the cache's own
    int *lengths_out;
    int *keep_idx;
    int keep_stride;
    PackedScales s;                      // s.k NULL: not in 4 bits
    int2 *plan;                     // [max_batch]: kept tokens (-1: leave the sequence), the first one that moves
    unsigned *keep;                 // [max_batch, capacity] slots of the kept tokens
    int *status;
};
cudaError_t launch_cache_evict(int row_bytes, const CacheEvictParams &p, cudaStream_t s);   // row_bytes: of a head of K or V

}  // namespace fz
