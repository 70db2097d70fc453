// sm_100a kernels of the embedding lookup and of its gradient.
//
// Lookup:    out[i] = scale * table[ids[i] - first_row], a row of zeros when that row is not in the table.
// Gradient:  g[v] = (accumulate ? g[v] : 0) + scale * sum over the tokens i with ids[i] - first_row = v of grad[i].
//
// Both only move data, so both are bound by HBM: the lookup reads and writes n rows, the gradient reads n rows and writes
// the whole table (the rows no token has get zeros in the same pass).  Sums are fp32 and rounded once at the end.
//
// Gradient.  Tokens are grouped by row, so that every row of the table is summed without floating-point atomics: the order of
// the additions, hence every bit of the result, depends on the ids alone.  The work list has items: a row and at most kChunk of
// its tokens, ascending.
//   up to kSmallTokens tokens: rank    every token counts, over all tokens, those of lower rows, of its row, and of its row before
//          it; that is its place in the list, and whether an item begins there.
//   more:  count   cnt[v] = number of tokens of row v; integer atomics, one per distinct row and warp
//          ranges  every row with tokens gets a range of the token list (where in the list does not matter) and its items
//          place   puts the tokens there, in order of arrival, which does depend on timing ...
//          sort    ... and in ascending order here: each token looks up how many of its row's tokens come before it; rows with
//                  more than kChunk tokens go through a bitmap of token positions in shared memory instead.
//   fill   zeros in the whole table.  It needs nothing of the above, so it runs beside it: beside rank, because it does not wait
//          for it; beside the others, because those go to a stream of the library's own, forked off and joined by events.  Of a large
//          table only a first part: the rest beside the sums, where the rows with tokens are known and left out.
//   sum    a group of threads per item and slab of columns adds up the gradients; a row with several items has them added in
//          ascending order by whichever group finishes last.
#include "rd_vocab.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <mutex>

#include "rd.h"
#include "rd_launch.h"
#include "rd_ptx.h"

namespace rd {

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kChunk = 32;         // tokens that one thread group adds up
constexpr uint32_t kBigItem = 8;        // items with more tokens are dealt out first, so that no thread group meets one at its end
constexpr uint32_t kSmallTokens = 4096; // up to here every token counts over all others (4096 tokens 9 us, 8000 tokens 33 us; the
                                        // sort of more takes 16 us)

template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float widen<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }

// V consecutive elements, at most 32 bytes of them, moved in one access.
template <typename T, int V> struct alignas(sizeof(T) * V) Vec {
    static_assert(sizeof(T) * V <= 32, "one access");
    T v[V];
};

template <typename T, int V> __device__ __forceinline__ Vec<T, V> load(const T *p)
{
    Vec<T, V> x;
    if constexpr (sizeof(x) == 32) {
        uint32_t(&w)[8] = *reinterpret_cast<uint32_t(*)[8]>(&x);
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                     : "l"(p));
    } else {
        x = *reinterpret_cast<const Vec<T, V> *>(p);
    }
    return x;
}
template <typename T, int V> __device__ __forceinline__ void store(T *p, const Vec<T, V> &x)
{
    if constexpr (sizeof(x) == 32) {
        const uint32_t(&w)[8] = *reinterpret_cast<const uint32_t(*)[8]>(&x);
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        *reinterpret_cast<Vec<T, V> *>(p) = x;
    }
}

// The table row of token i, or a negative number when the table does not hold it.
__device__ __forceinline__ long long row_of(const void *ids, bool wide, size_t i, long long first, size_t rows)
{
    const long long id = wide ? static_cast<const long long *>(ids)[i] : static_cast<const int *>(ids)[i];
    if (id < first) return -1;                   // first >= 0: negative ids too
    return id - first < static_cast<long long>(rows) ? id - first : -1;
}

constexpr int kGatherUnroll = 2;

// A thread block copies kThreads * kGatherUnroll consecutive vectors of the flattened output.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) rd_embed_kernel(const T *__restrict__ table, size_t table_stride, size_t rows, const void *__restrict__ ids,
                                                            bool wide, long long first, uint32_t vecs, size_t total, float scale,
                                                            T *__restrict__ out, size_t out_stride)
{
    pdl_start();
    const size_t base = size_t(blockIdx.x) * (kThreads * kGatherUnroll);
    const size_t row0 = base / vecs;
    const uint32_t off0 = uint32_t(base - row0 * vecs);
    Vec<T, V> x[kGatherUnroll];
    T *dst[kGatherUnroll];
#pragma unroll
    for (int u = 0; u < kGatherUnroll; u++) {
        const uint32_t o = off0 + u * kThreads + threadIdx.x;
        dst[u] = nullptr;
        if (base + u * kThreads + threadIdx.x >= total) continue;
        const size_t i = row0 + o / vecs;
        const uint32_t j = o % vecs;
        dst[u] = out + i * out_stride + size_t(j) * V;
        const long long r = row_of(ids, wide, i, first, rows);
        if (r >= 0) {
            x[u] = load<T, V>(table + size_t(r) * table_stride + size_t(j) * V);
        } else {
#pragma unroll
            for (int k = 0; k < V; k++) x[u].v[k] = narrow<T>(0.0f);
        }
    }
#pragma unroll
    for (int u = 0; u < kGatherUnroll; u++) {
        if (!dst[u]) continue;
        if (scale != 1.0f) {
#pragma unroll
            for (int k = 0; k < V; k++) x[u].v[k] = narrow<T>(widen<T>(x[u].v[k]) * scale);
        }
        store<T, V>(dst[u], x[u]);
    }
}

// Rows that are not made of 16-byte words: a warp per kRowUnroll * 32 elements of a row, single elements side by side.  (With
// elements dealt out like the vectors above, the divisions took most of the time: 16384 rows of 1001 bf16 values 52 us, this 12.)
constexpr int kRowUnroll = 16;
template <typename T>
__global__ void __launch_bounds__(kThreads) rd_embed_element_kernel(const T *__restrict__ table, size_t table_stride, size_t rows, const void *__restrict__ ids,
                                                                    bool wide, long long first, uint32_t dim, uint32_t slabs, size_t units, float scale,
                                                                    T *__restrict__ out, size_t out_stride)
{
    pdl_start();
    const int lane = threadIdx.x & 31;
    const size_t u = size_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
    if (u >= units) return;
    const size_t i = u / slabs;
    const uint32_t j = uint32_t(u - i * slabs) * (32 * kRowUnroll) + lane;
    const long long r = row_of(ids, wide, i, first, rows);
    const T *src = table + (r >= 0 ? size_t(r) * table_stride : 0) + j;
    T *dst = out + i * out_stride + j;
    T x[kRowUnroll];
#pragma unroll
    for (int e = 0; e < kRowUnroll; e++) x[e] = r >= 0 && j + 32 * e < dim ? src[32 * e] : narrow<T>(0.0f);
#pragma unroll
    for (int e = 0; e < kRowUnroll; e++)
        if (j + 32 * e < dim) dst[32 * e] = scale != 1.0f && r >= 0 ? narrow<T>(widen<T>(x[e]) * scale) : x[e];
}

template <typename T> cudaError_t launch_elements(const EmbedArgs &a)
{
    const uint32_t slabs = uint32_t((a.dim + 32 * kRowUnroll - 1) / (32 * kRowUnroll));
    const size_t units = a.n * slabs, blocks = (units + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffffu) return cudaErrorInvalidConfiguration;
    return launch(rd_embed_element_kernel<T>, unsigned(blocks), kThreads, a.stream, static_cast<const T *>(a.table), a.table_stride, a.rows, a.ids, a.wide_ids, a.first_row,
                  uint32_t(a.dim), slabs, units, a.scale, static_cast<T *>(a.out), a.out_stride);
}

template <typename T, int V> cudaError_t launch_embed(const EmbedArgs &a)
{
    const uint32_t vecs = uint32_t(a.dim / V);
    const size_t total = a.n * vecs;
    const size_t per = size_t(kThreads) * kGatherUnroll;
    const size_t blocks = (total + per - 1) / per;
    if (blocks > 0x7fffffffu) return cudaErrorInvalidConfiguration;
    return launch(rd_embed_kernel<T, V>, unsigned(blocks), kThreads, a.stream, static_cast<const T *>(a.table), a.table_stride, a.rows, a.ids, a.wide_ids, a.first_row,
                  vecs, total, a.scale, static_cast<T *>(a.out), a.out_stride);
}

// Whether rows begin and end on multiples of `to` bytes.
bool vector_rows(const void *p, size_t stride, size_t dim, size_t esize, size_t to)
{
    return reinterpret_cast<uintptr_t>(p) % to == 0 && stride * esize % to == 0 && dim * esize % to == 0;
}

// ---------------------------------------------------------------------------------------------------- gradient

struct GradMeta {
    uint32_t list_used;       // entries of the token list handed out to rows
    uint32_t n_big;           // items with more than kBigItem tokens: items[0 ..
    uint32_t n_items;         // the others, from items[big_room] on; some may be empty
    uint32_t n_long;          // rows with more than kChunk tokens
};

struct Item {
    uint32_t row, begin, count;       // list[begin .. begin + count)
    uint32_t part, parts;             // which of the row's items this is, and how many there are
    uint32_t pad;
};

// Where the partial sums of part k of a row go whose tokens begin at list[begin]: no two parts of rows with more than kChunk tokens
// get the same one, since of kChunk consecutive list entries at most one begins a first part and at most one a later one.
__host__ __device__ __forceinline__ uint32_t slot_of(uint32_t begin, uint32_t k) { return 2 * ((begin + k * kChunk) / kChunk) + (k == 0); }

struct GradWork {             // the workspace's parts
    GradMeta *meta;
    uint32_t *cnt;            // rows
    uint32_t *start;          // rows: where the row's tokens begin in the list
    uint32_t *rank;           // n: arrival number of the token within its row
    uint32_t *arrived;        // n: token list, in order of arrival within a row
    uint32_t *list;           // n: token list, ascending within a row
    uint32_t *long_row;       // rows with more than kChunk tokens
    Item *items;
    uint32_t *done;           // per slot and slab: items of the row that have their partial sums written
    float *partial;           // per slot: dim fp32 values
    uint32_t big_room;
    size_t partial_stride, bytes, zero_bytes;
};

constexpr unsigned kSumBlocks = 148 * 3;
constexpr uint32_t kMostLanes = 32;       // threads per item and slab: within a warp
size_t max_long(size_t n) { return n / (kChunk + 1); }
size_t max_slots(size_t n) { return n > kChunk ? 2 * (n / kChunk + 1) : 0; }
size_t max_big(size_t n) { return n <= kSmallTokens ? 0 : n / (kBigItem + 1); }
size_t max_items(size_t n, size_t rows) { return n <= kSmallTokens ? n : (n < rows ? n : rows) + n / kChunk; }
uint32_t lanes_for(uint32_t vecs)
{
    uint32_t lanes = 8;
    while (lanes < kMostLanes && lanes < vecs) lanes *= 2;
    return lanes;
}
// Slabs of columns when a thread moves one element at a time: the most there can be.
size_t max_slabs(size_t dim) { return (dim + kMostLanes - 1) / kMostLanes; }

GradWork layout(void *workspace, size_t rows, size_t dim, size_t n)
{
    GradWork w{};
    size_t at = 0;
    char *base = static_cast<char *>(workspace);
    auto take = [&](size_t bytes) {
        char *p = base + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    const bool small = n <= kSmallTokens;
    w.partial_stride = (dim + 7) / 8 * 8;
    w.meta = reinterpret_cast<GradMeta *>(take(sizeof(GradMeta)));
    if (!small) {
        w.cnt = reinterpret_cast<uint32_t *>(take(rows * 4));
        w.zero_bytes = at;
        w.start = reinterpret_cast<uint32_t *>(take(rows * 4));
        w.rank = reinterpret_cast<uint32_t *>(take(n * 4));
        w.arrived = reinterpret_cast<uint32_t *>(take(n * 4));
        w.long_row = reinterpret_cast<uint32_t *>(take(max_long(n) * 4));
    }
    w.list = reinterpret_cast<uint32_t *>(take(n * 4));
    w.big_room = uint32_t(max_big(n));
    w.items = reinterpret_cast<Item *>(take((max_big(n) + max_items(n, rows)) * sizeof(Item)));
    w.done = reinterpret_cast<uint32_t *>(take(max_slots(n) * max_slabs(dim) * 4));
    w.partial = reinterpret_cast<float *>(take(max_slots(n) * w.partial_stride * 4));
    w.bytes = at;
    return w;
}

__global__ void __launch_bounds__(kThreads) rd_embed_count_kernel(const void *__restrict__ ids, bool wide, long long first, size_t rows, uint32_t n,
                                                                  uint32_t *__restrict__ cnt, uint32_t *__restrict__ rank)
{
    pdl_wait_first();
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    const long long r = i < n ? row_of(ids, wide, i, first, rows) : -1;
    // lanes with the same row count together: one atomic each
    const uint32_t key = r >= 0 ? uint32_t(r) : 0xffffffffu;
    const uint32_t peers = __match_any_sync(0xffffffffu, key);
    const int lane = threadIdx.x & 31, leader = __ffs(peers) - 1;
    uint32_t base = 0;
    if (r >= 0 && lane == leader) base = atomicAdd(&cnt[r], uint32_t(__popc(peers)));
    base = __shfl_sync(0xffffffffu, base, leader);
    if (i < n) rank[i] = base + __popc(peers & ((1u << lane) - 1));
}

// Inclusive sum over a thread block of 1024; `total` is the whole block's.  Two barriers; `shared` has 33 words.
__device__ __forceinline__ uint32_t block_sum(uint32_t x, uint32_t *shared, uint32_t &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += o;
    }
    __syncthreads();
    if (lane == 31) shared[warp] = x;
    __syncthreads();
    uint32_t s = shared[lane];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += o;
    }
    total = __shfl_sync(0xffffffffu, s, 31);
    const uint32_t before = __shfl_sync(0xffffffffu, s, warp ? warp - 1 : 0);
    return x + (warp ? before : 0);
}

// Hands every row a range of the token list, its items and their partial rows: those of a thread block's rows follow each other.
__global__ void __launch_bounds__(1024) rd_embed_ranges_kernel(GradWork w, size_t rows, uint32_t slabs)
{
    __shared__ uint32_t shared[32];
    __shared__ uint32_t bases[3];
    pdl_start();
    const size_t v = size_t(blockIdx.x) * 1024 + threadIdx.x;
    const uint32_t c = v < rows ? w.cnt[v] : 0;
    const uint32_t parts = (c + kChunk - 1) / kChunk;
    const uint32_t last = c - (parts ? parts - 1 : 0) * kChunk;          // tokens of the last part; the others have kChunk
    const uint32_t n_big = parts ? parts - (last <= kBigItem) : 0;
    uint32_t all_tokens, all_big, all_items;
    const uint32_t tokens = block_sum(c, shared, all_tokens) - c;
    const uint32_t big = block_sum(n_big, shared, all_big) - n_big;
    const uint32_t items = block_sum(parts - n_big, shared, all_items) - (parts - n_big);
    if (threadIdx.x == 0) {
        bases[0] = all_tokens ? atomicAdd(&w.meta->list_used, all_tokens) : 0;
        bases[1] = all_big ? atomicAdd(&w.meta->n_big, all_big) : 0;
        bases[2] = all_items ? atomicAdd(&w.meta->n_items, all_items) : 0;
    }
    __syncthreads();
    if (c == 0) return;
    const uint32_t begin = bases[0] + tokens;
    w.start[v] = begin;
    for (uint32_t k = 0; k < n_big; k++) w.items[bases[1] + big + k] = Item{uint32_t(v), begin + k * kChunk, min(kChunk, c - k * kChunk), k, parts, 0};
    if (n_big < parts) w.items[w.big_room + bases[2] + items] = Item{uint32_t(v), begin + n_big * kChunk, last, n_big, parts, 0};
    if (parts > 1) {
        w.long_row[atomicAdd(&w.meta->n_long, 1u)] = uint32_t(v);
        for (uint32_t k = 0; k < slabs; k++) w.done[size_t(slot_of(begin, 0)) * slabs + k] = 0;
    }
}

// All of it for few tokens: a warp per token counts over all of them.
__global__ void __launch_bounds__(1024) rd_embed_rank_kernel(const void *__restrict__ ids, bool wide, long long first, size_t rows, uint32_t n, GradWork w, uint32_t slabs)
{
    __shared__ __align__(16) uint32_t row[kSmallTokens];
    pdl_wait_first();
    const int lane = threadIdx.x & 31;
    const uint32_t padded = (n + 127) / 128 * 128, i = blockIdx.x * 32 + (threadIdx.x >> 5);
    for (uint32_t k = threadIdx.x; k < padded; k += 1024) {
        const long long r = k < n ? row_of(ids, wide, k, first, rows) : -1;
        row[k] = r >= 0 ? uint32_t(r) : 0xffffffffu;          // tokens of other slices come last
    }
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.meta = GradMeta{0, 0, n, 0};
    if (i >= n) return;
    const uint32_t mine = row[i];
    uint32_t lower = 0, same = 0, before = 0;
    for (uint32_t k = 4 * lane; k < padded; k += 128) {
        const uint4 x = *reinterpret_cast<const uint4 *>(row + k);
        const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int u = 0; u < 4; u++) {
            lower += v[u] < mine;
            same += v[u] == mine;
            before += v[u] == mine && k + u < i;
        }
    }
    lower = __reduce_add_sync(0xffffffffu, lower);
    same = __reduce_add_sync(0xffffffffu, same);
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane) return;
    const uint32_t at = lower + before, parts = (same + kChunk - 1) / kChunk;
    const bool here = mine != 0xffffffffu, opens = here && before % kChunk == 0;
    if (here) w.list[at] = i;
    w.items[at] = Item{mine, at, opens ? min(kChunk, same - before) : 0, before / kChunk, parts, 0};
    if (opens && before == 0 && parts > 1)
        for (uint32_t k = 0; k < slabs; k++) w.done[size_t(slot_of(at, 0)) * slabs + k] = 0;
}

__global__ void __launch_bounds__(kThreads) rd_embed_place_kernel(const void *__restrict__ ids, bool wide, long long first, size_t rows, uint32_t n,
                                                                  const uint32_t *__restrict__ start, const uint32_t *__restrict__ rank, uint32_t *__restrict__ arrived)
{
    pdl_start();
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= n) return;
    const long long r = row_of(ids, wide, i, first, rows);
    if (r >= 0) arrived[start[r] + rank[i]] = i;
}

constexpr uint32_t kBitmapWords = 8192;      // 32 KB of shared memory: 262144 token positions per sweep

// Thread blocks below token_blocks: one thread per token of a row with at most kChunk tokens.  The others: rows with more.
__global__ void __launch_bounds__(kThreads) rd_embed_sort_kernel(const void *__restrict__ ids, bool wide, long long first, size_t rows, uint32_t n,
                                                                 const uint32_t *__restrict__ cnt, const uint32_t *__restrict__ start,
                                                                 const uint32_t *__restrict__ arrived, uint32_t *__restrict__ list, const GradMeta *meta,
                                                                 const uint32_t *__restrict__ long_row, uint32_t token_blocks)
{
    pdl_start();
    __shared__ uint32_t bits[kBitmapWords];
    __shared__ uint32_t warp_sum[kThreads / 32];
    if (blockIdx.x < token_blocks) {
        const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
        if (i >= n) return;
        const long long r = row_of(ids, wide, i, first, rows);
        if (r < 0) return;
        const uint32_t c = cnt[r], s = start[r];
        if (c > kChunk) return;
        uint32_t before = 0;
        for (uint32_t k = 0; k < c; k++) before += arrived[s + k] < i;
        list[s + before] = i;
        return;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint32_t q = blockIdx.x - token_blocks; q < meta->n_long; q += gridDim.x - token_blocks) {
        const uint32_t r = long_row[q], c = cnt[r], s = start[r];
        uint32_t done = 0;                       // tokens written
        for (uint64_t from = 0; from < n; from += uint64_t(kBitmapWords) * 32) {
            const uint64_t words64 = (n - from + 31) / 32;
            const uint32_t words = words64 < kBitmapWords ? uint32_t(words64) : kBitmapWords;
            for (uint32_t w = threadIdx.x; w < words; w += kThreads) bits[w] = 0;
            __syncthreads();
            for (uint32_t k = threadIdx.x; k < c; k += kThreads) {
                const uint64_t p = arrived[s + k];
                if (p >= from && p - from < uint64_t(words) * 32) atomicOr(&bits[uint32_t(p - from) >> 5], 1u << (uint32_t(p - from) & 31));
            }
            __syncthreads();
            for (uint32_t w0 = 0; w0 < words; w0 += kThreads) {
                const uint32_t w = w0 + threadIdx.x;
                uint32_t b = w < words ? bits[w] : 0;
                uint32_t incl = __popc(b);
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const uint32_t o = __shfl_up_sync(0xffffffffu, incl, d);
                    if (lane >= d) incl += o;
                }
                if (lane == 31) warp_sum[warp] = incl;
                __syncthreads();
                uint32_t at = done + incl - __popc(b), all = 0;
#pragma unroll
                for (int k = 0; k < kThreads / 32; k++) {
                    if (k < warp) at += warp_sum[k];
                    all += warp_sum[k];
                }
                for (; b; b &= b - 1) list[s + at++] = uint32_t(from + uint64_t(w) * 32 + __ffs(b) - 1);
                done += all;
                __syncthreads();
            }
        }
    }
}

// A thread's V columns: vectors of consecutive ones, or for rows that are not made of 16-byte words (ELEMENTS) single ones that are
// `step` apart, so that neighbouring lanes have neighbouring columns; `left` of them, counted from the first, exist.
template <int V, bool ELEMENTS> struct Columns {
    uint32_t step, left;
    template <typename T> __device__ __forceinline__ Vec<T, V> get(const T *p) const
    {
        if constexpr (!ELEMENTS) {
            return load<T, V>(p);
        } else {
            Vec<T, V> x;
#pragma unroll
            for (int e = 0; e < V; e++) x.v[e] = e * step < left ? p[e * step] : narrow<T>(0.0f);
            return x;
        }
    }
    template <typename T> __device__ __forceinline__ void put(T *p, const Vec<T, V> &x) const
    {
        if constexpr (!ELEMENTS) {
            store<T, V>(p, x);
        } else {
#pragma unroll
            for (int e = 0; e < V; e++)
                if (e * step < left) p[e * step] = x.v[e];
        }
    }
};

// Sum over c tokens, in order, several of them in flight.  The tokens are in the lanes of the warp (token t in lane t) or, for groups
// narrower than a warp, in list.
template <typename T, int V, bool ELEMENTS>
__device__ __forceinline__ void add_rows(const Columns<V, ELEMENTS> &cols, const T *__restrict__ grad, size_t stride, uint32_t token, const uint32_t *__restrict__ list,
                                         uint32_t c, float (&acc)[V])
{
    constexpr int U = ELEMENTS ? 2 : 4;
    auto row = [&](uint32_t t) { return cols.get(grad + size_t(list ? list[t] : __shfl_sync(0xffffffffu, token, t)) * stride); };
#pragma unroll
    for (int k = 0; k < V; k++) acc[k] = 0.0f;
    uint32_t t = 0;
    for (; t + U <= c; t += U) {
        Vec<T, V> x[U];
#pragma unroll
        for (int u = 0; u < U; u++) x[u] = row(t + u);
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int k = 0; k < V; k++) acc[k] += widen<T>(x[u].v[k]);
    }
    for (; t < c; t++) {
        const Vec<T, V> x = row(t);
#pragma unroll
        for (int k = 0; k < V; k++) acc[k] += widen<T>(x.v[k]);
    }
}

template <typename O, int V, bool ELEMENTS>
__device__ __forceinline__ void write_row(const Columns<V, ELEMENTS> &cols, O *p, const float (&acc)[V], float scale, bool accumulate)
{
    Vec<O, V> y;
    if (accumulate) {
        const Vec<O, V> old = cols.get(static_cast<const O *>(p));
#pragma unroll
        for (int k = 0; k < V; k++) y.v[k] = narrow<O>(fmaf(acc[k], scale, widen<O>(old.v[k])));
    } else {
#pragma unroll
        for (int k = 0; k < V; k++) y.v[k] = narrow<O>(acc[k] * scale);
    }
    cols.put(p, y);
}

// `lanes` threads (a power of two, within a warp) work on an item and a slab of lanes * V columns.  An item, its tokens and their
// rows are three loads that depend on each other; the item after the next one and the next one's tokens are on their way
// while a group adds up the rows of the present one.
template <typename T, typename O, int V, bool ELEMENTS>
__global__ void __launch_bounds__(kThreads, 3) rd_embed_sum_kernel(const T *__restrict__ grad, size_t grad_stride, O *__restrict__ table, size_t table_stride, uint32_t dim,
                                                                uint32_t lanes, uint32_t slabs, float scale, bool accumulate, GradWork w)
{
    pdl_start();
    const uint32_t per_block = kThreads / lanes, lane = threadIdx.x % lanes, group = threadIdx.x / lanes;
    const uint32_t mask = (lanes == 32 ? 0xffffffffu : (1u << lanes) - 1) << (threadIdx.x % 32 / lanes * lanes);     // the group within its warp
    const uint32_t n_big = w.meta->n_big, others = w.big_room - n_big;
    const uint64_t units = (uint64_t(n_big) + w.meta->n_items) * slabs, step = uint64_t(gridDim.x) * per_block;
    const bool by_lane = lanes == 32;
    auto item = [&](uint64_t u) {
        if (u >= units) return Item{};
        const size_t k = u / slabs;
        return w.items[k < n_big ? k : k + others];
    };
    auto tokens = [&](const Item &it) { return by_lane && lane < it.count ? w.list[it.begin + lane] : 0; };
    uint64_t u = uint64_t(blockIdx.x) * per_block + group;
    Item it = item(u), next = item(u + step);
    uint32_t token = tokens(it);
    for (; u < units; u += step) {
        const Item after = item(u + 2 * step);
        const uint32_t next_token = tokens(next);
        if (it.count) {
            const uint32_t slab = uint32_t(u % slabs), at = slab * lanes * V + (ELEMENTS ? lane : lane * V);
            const bool mine = at < dim;
            const size_t col = mine ? at : 0;                     // lanes beyond the row read its beginning and write nothing
            const Columns<V, ELEMENTS> cols{lanes, mine ? dim - at : 0};
            float acc[V];
            add_rows(cols, grad + col, grad_stride, token, by_lane ? nullptr : w.list + it.begin, it.count, acc);
            O *out = table + size_t(it.row) * table_stride + col;
            if (it.parts == 1) {
                if (mine) write_row(cols, out, acc, scale, accumulate);
            } else {
                // a row of several items: whichever group is last adds the partial rows up, in order
                const uint32_t begin = it.begin - it.part * kChunk;
                float *partial = w.partial + col;
                if (mine) {
                    Vec<float, V> x;
#pragma unroll
                    for (int e = 0; e < V; e++) x.v[e] = acc[e];
                    cols.put(partial + size_t(slot_of(begin, it.part)) * w.partial_stride, x);
                }
                __threadfence();
                __syncwarp(mask);
                uint32_t finished = lane == 0 ? atomicAdd(&w.done[size_t(slot_of(begin, 0)) * slabs + slab], 1u) + 1 : 0;
                finished = __shfl_sync(mask, finished, 0, lanes);
                if (finished == it.parts && mine) {
                    __threadfence();
#pragma unroll
                    for (int e = 0; e < V; e++) acc[e] = 0.0f;
#pragma unroll 4
                    for (uint32_t k = 0; k < it.parts; k++) {
                        const Vec<float, V> x = cols.get(const_cast<const float *>(partial) + size_t(slot_of(begin, k)) * w.partial_stride);
#pragma unroll
                        for (int e = 0; e < V; e++) acc[e] += x.v[e];
                    }
                    write_row(cols, out, acc, scale, accumulate);
                }
            }
        }
        it = next;
        next = after;
        token = next_token;
    }
}

// The same for rows of whole 16-byte words from kStreamBytes on: the gradients' rows come through shared memory by bulk copies, so
// that a warp has up to 12 KB on its way whatever the items look like (through registers a warp had the 1 to 4 KB of one item; when
// the whole table was filled before: the gradient of 16384 tokens x 4096 bf16 into 131072 rows 216 us, this 201; of 65536 tokens into a slice of 32768 x 2048 92, 77.
// 8 warps with 24 KB each: 207, 81; 24 with 8 KB: 201, 81; 32 with 6 KB: 208, 95).
//   A warp takes 32 items at a time, one per lane, and sees their tokens as one sequence.  Lanes look up 32 tokens of it at a
//   time; groups of 4 are copied to a ring of 3 groups, two groups ahead of the one that is added up.
constexpr int kGroup = 4, kGroups = 3;
constexpr uint32_t kSlab = 1024;          // bytes of a row that a warp takes: two words of 16 bytes per lane, 512 apart
constexpr size_t kStreamBytes = 512;
constexpr int kStreamThreads = 512;
constexpr uint32_t kStreamSmem = kStreamThreads / 32 * (kGroups * kGroup * kSlab) + 128;

__device__ int g_embed_status;

template <typename T, typename O>
__global__ void __launch_bounds__(kStreamThreads, 1) rd_embed_stream_kernel(const T *__restrict__ grad, size_t grad_stride, O *__restrict__ table, size_t table_stride,
                                                                            uint32_t dim, uint32_t slabs, float scale, bool accumulate, GradWork w)
{
    constexpr uint32_t V = 16 / sizeof(T), kWords = kSlab / 16 / 32, kColumns = kSlab / sizeof(T);
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) unsigned long long bars[kStreamThreads / 32][kGroups];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t slots = smem_addr(ring) + warp * (kGroups * kGroup * kSlab), bar0 = smem_addr(&bars[warp][0]);
    if (lane < kGroups) bar_init(bar0 + 8 * lane, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    pdl_start();
    const uint32_t n_big = w.meta->n_big, others = w.big_room - n_big;
    const uint64_t units = (uint64_t(n_big) + w.meta->n_items) * slabs, step = uint64_t(gridDim.x) * (kStreamThreads / 32);
    uint32_t sent = 0;                                       // groups since the kernel began
    for (uint64_t first = uint64_t(blockIdx.x) * (kStreamThreads / 32) + warp; first < units; first += 32 * step) {
        // a lane's item, its slab, and where its tokens lie in the sequence
        const uint64_t u = first + lane * step;
        Item it{};
        if (u < units) {
            const size_t k = u / slabs;
            it = w.items[k < n_big ? k : k + others];
        }
        const uint32_t slab = uint32_t(u % slabs);
        uint32_t upto = it.count;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        const uint32_t total = __shfl_sync(0xffffffffu, upto, 31), groups = (total + kGroup - 1) / kGroup, sent0 = sent;
        const T *src = nullptr;
        uint32_t bytes = 0;
        int cur = -1;                                        // the item being added up, and its tokens that are left
        uint32_t left = 0;
        float acc[kWords][V];
        for (uint32_t g = 0; g < groups + 2; g++) {
            if (g < groups) {
                if (g % (32 / kGroup) == 0) {
                    // the next 32 tokens: whose they are, and their rows
                    const uint32_t f = g * kGroup + lane;
                    uint32_t owner = 0;                      // the first item that reaches beyond f
#pragma unroll
                    for (int d = 16; d; d /= 2)
                        if (__shfl_sync(0xffffffffu, upto, owner + d - 1) <= f) owner += d;
                    owner &= 31;
                    const uint32_t begin = __shfl_sync(0xffffffffu, it.begin, owner), before = __shfl_sync(0xffffffffu, upto - it.count, owner);
                    const uint32_t col = __shfl_sync(0xffffffffu, slab, owner) * kColumns;
                    bytes = 0;
                    if (f < total) {
                        src = grad + size_t(w.list[begin + f - before]) * grad_stride + col;
                        bytes = min(kSlab, uint32_t((dim - col) * sizeof(T)));
                    }
                }
                const bool mine = uint32_t(lane) / kGroup == g % (32 / kGroup);
                const uint32_t all = __reduce_add_sync(0xffffffffu, mine ? bytes : 0), s = sent % kGroups, bar = bar0 + 8 * s;
                if (lane == 0) bar_expect(bar, all);
                __syncwarp();
                if (mine && bytes)
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(slots + (s * kGroup + lane % kGroup) * kSlab),
                                 "l"(src), "r"(bytes), "r"(bar)
                                 : "memory");
                sent++;
            }
            if (g < 2) continue;
            // the group two back
            const uint32_t t0 = (g - 2) * kGroup, G = sent0 + g - 2, s = G % kGroups, parity = G / kGroups & 1, bar = bar0 + 8 * s;
            if (!__all_sync(0xffffffffu, bar_try(bar, parity))) {
                const long long began = clock64();
                bool done = false;
                do done = __all_sync(0xffffffffu, bar_try(bar, parity));
                while (!done && __any_sync(0xffffffffu, clock64() - began < kWaitCycles));
                if (!done) {
                    atomicExch(&g_embed_status, 1);
                    drain();
                    return;
                }
            }
            for (int t = 0; t < kGroup && t0 + t < total; t++) {
                if (left == 0) {
                    do left = __shfl_sync(0xffffffffu, it.count, ++cur);
                    while (left == 0);
#pragma unroll
                    for (uint32_t h = 0; h < kWords; h++)
#pragma unroll
                        for (uint32_t e = 0; e < V; e++) acc[h][e] = 0.0f;
                }
#pragma unroll
                for (uint32_t h = 0; h < kWords; h++) {
                    Vec<T, V> x;
                    uint32_t(&b)[4] = *reinterpret_cast<uint32_t(*)[4]>(&x);
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3])
                                 : "r"(slots + (s * kGroup + t) * kSlab + h * 512 + lane * 16)
                                 : "memory");
#pragma unroll
                    for (uint32_t e = 0; e < V; e++) acc[h][e] += widen<T>(x.v[e]);
                }
                if (--left) continue;
                // the item is complete
                const uint32_t row = __shfl_sync(0xffffffffu, it.row, cur), part = __shfl_sync(0xffffffffu, it.part, cur), parts = __shfl_sync(0xffffffffu, it.parts, cur);
                const uint32_t begin = __shfl_sync(0xffffffffu, it.begin, cur) - part * kChunk, at_slab = __shfl_sync(0xffffffffu, slab, cur);
                const uint32_t col0 = at_slab * kColumns + lane * V;
                const Columns<int(V), false> cols{0, 0};
                bool write = parts == 1;
                if (parts > 1) {
#pragma unroll
                    for (uint32_t h = 0; h < kWords; h++) {
                        Vec<float, V> x;
#pragma unroll
                        for (uint32_t e = 0; e < V; e++) x.v[e] = acc[h][e];
                        if (col0 + h * 32 * V < dim) store<float, V>(w.partial + size_t(slot_of(begin, part)) * w.partial_stride + col0 + h * 32 * V, x);
                    }
                    __threadfence();
                    __syncwarp();
                    uint32_t finished = lane == 0 ? atomicAdd(&w.done[size_t(slot_of(begin, 0)) * slabs + at_slab], 1u) + 1 : 0;
                    finished = __shfl_sync(0xffffffffu, finished, 0);
                    write = finished == parts;
                    if (write) {
                        // whichever warp is last adds the row's partial sums up, in order
                        __threadfence();
#pragma unroll
                        for (uint32_t h = 0; h < kWords; h++)
#pragma unroll
                            for (uint32_t e = 0; e < V; e++) acc[h][e] = 0.0f;
                        constexpr uint32_t kAhead = 4;       // partial sums on their way
                        for (uint32_t k0 = 0; k0 < parts; k0 += kAhead) {
                            Vec<float, V> x[kAhead][kWords];
#pragma unroll
                            for (uint32_t k = 0; k < kAhead; k++)
#pragma unroll
                                for (uint32_t h = 0; h < kWords; h++)
                                    if (k0 + k < parts && col0 + h * 32 * V < dim)
                                        x[k][h] = load<float, V>(w.partial + size_t(slot_of(begin, k0 + k)) * w.partial_stride + col0 + h * 32 * V);
#pragma unroll
                            for (uint32_t k = 0; k < kAhead; k++)
#pragma unroll
                                for (uint32_t h = 0; h < kWords; h++)
#pragma unroll
                                    for (uint32_t e = 0; e < V; e++) acc[h][e] += k0 + k < parts && col0 + h * 32 * V < dim ? x[k][h].v[e] : 0.0f;
                        }
                    }
                }
                if (write) {
#pragma unroll
                    for (uint32_t h = 0; h < kWords; h++)
                        if (col0 + h * 32 * V < dim) write_row(cols, table + size_t(row) * table_stride + col0 + h * 32 * V, acc[h], scale, accumulate);
                }
            }
            __syncwarp();                                    // everyone has read the group's slots before they are filled again
        }
    }
}

// Zeros.  Thread blocks of a plain grid write 16 KB each, one after the other in memory: at 7.4 TB/s against 6.3 TB/s when the
// blocks of a resident grid stride over the table (1 GiB, B200), whose stores drift apart.
constexpr uint32_t kFillBytes = 16384;

__device__ __forceinline__ void fill_span(char *p, size_t bytes, uint32_t t, uint32_t threads)
{
    // single elements up to a 32-byte boundary and behind the last one
    const size_t head = (32 - reinterpret_cast<uintptr_t>(p) % 32) % 32, h = head < bytes ? head : bytes;
    for (size_t i = 2 * t; i < h; i += 2 * threads) *reinterpret_cast<uint16_t *>(p + i) = 0;
    p += h;
    bytes -= h;
    const size_t wide = bytes / 32 * 32;
    for (size_t i = size_t(t) * 32; i < wide; i += size_t(threads) * 32)
        asm volatile("st.global.v8.b32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"l"(p + i), "r"(0) : "memory");
    for (size_t i = wide + 2 * t; i < bytes; i += 2 * threads) *reinterpret_cast<uint16_t *>(p + i) = 0;
}

// The same for 16 KB of a table whose rows follow each other without gaps, except rows with tokens.  Everything is made of units of
// `unit` bytes (16 or 32), which lie within a row.
__device__ __forceinline__ void fill_empty(char *table, size_t span, uint32_t row_bytes, const uint32_t *__restrict__ cnt, uint32_t unit)
{
    const size_t from = size_t(blockIdx.x) * kFillBytes, row0 = from / row_bytes;
    const uint32_t in_row = uint32_t(from - row0 * row_bytes), bytes = uint32_t(span - from < kFillBytes ? span - from : kFillBytes);
    for (uint32_t i = threadIdx.x * unit; i < bytes; i += kThreads * unit) {
        if (__ldg(cnt + row0 + (in_row + i) / row_bytes)) continue;
        if (unit == 32) asm volatile("st.global.v8.b32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"l"(table + from + i), "r"(0) : "memory");
        else *reinterpret_cast<uint4 *>(table + from + i) = make_uint4(0, 0, 0, 0);
    }
}

// span > 0: the table is one piece of memory of that many bytes.  Otherwise rows of row_bytes, pitch apart, a warp each.
// cnt: tokens of every row; rows that have some are left alone.  Null: all rows.
// Only the last thread block waits for the kernels before: what comes after this kernel then comes after them too.  That the
// stream's earlier work is done is known from the first of them, which waits for it before it lets anything follow.
__global__ void __launch_bounds__(kThreads) rd_embed_fill_kernel(char *__restrict__ table, size_t span, size_t rows, size_t row_bytes, size_t pitch,
                                                                 const uint32_t *__restrict__ cnt, bool alone)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (alone || blockIdx.x == gridDim.x - 1) asm volatile("griddepcontrol.wait;" ::: "memory");
    if (span && cnt) {
        if (size_t(blockIdx.x) * kFillBytes < span)
            fill_empty(table, span, uint32_t(row_bytes), cnt, (reinterpret_cast<uintptr_t>(table) | row_bytes) % 32 ? 16 : 32);
    } else if (span) {
        const size_t from = size_t(blockIdx.x) * kFillBytes;
        // cut at addresses that are multiples of 32 bytes
        const size_t skew = reinterpret_cast<uintptr_t>(table) % 32;
        const size_t begin = blockIdx.x ? from - skew : 0, end = from + kFillBytes - skew;
        if (begin < span) fill_span(table + begin, (end < span ? end : span) - begin, threadIdx.x, kThreads);
    } else {
        const size_t row = size_t(blockIdx.x) * (kThreads / 32) + threadIdx.x / 32;
        if (row < rows && !(cnt && cnt[row])) fill_span(table + row * pitch, row_bytes, threadIdx.x % 32, 32);
    }
}

// A stream and four events of the library's own per device, made on the first call that wants them and kept.  Calls take turns to
// enqueue, so the events always stand for the call that holds the lock.
struct Lane {
    bool tried = false, ready = false;
    unsigned long long user = 0;              // the stream of the last call
    cudaStream_t side = nullptr;
    cudaEvent_t fork = nullptr, sorted = nullptr, filled = nullptr, join = nullptr;
};
constexpr int kMaxDevices = 64;
Lane g_lane[kMaxDevices];
std::mutex g_lane_mutex;

// Null where everything has to stay on the caller's stream: no such stream to be had, the call is being recorded into a graph, or
// another stream's call is still under way on it, which this one must not wait for.
Lane *lane_for(cudaStream_t stream)
{
    int device = 0;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    unsigned long long user = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device >= kMaxDevices) return nullptr;
    if (cudaStreamIsCapturing(stream, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone) return nullptr;
    if (cudaStreamGetId(stream, &user) != cudaSuccess) return nullptr;
    // what follows is no part of a recording that another thread may be at
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    if (cudaThreadExchangeStreamCaptureMode(&mode) != cudaSuccess) return nullptr;
    Lane &l = g_lane[device];
    if (!l.tried) {
        l.tried = true;
        // of the highest priority: its few thread blocks go ahead of the many of the fill that are queued already
        int lowest = 0, highest = 0;
        l.ready = cudaDeviceGetStreamPriorityRange(&lowest, &highest) == cudaSuccess &&
                  cudaStreamCreateWithPriority(&l.side, cudaStreamNonBlocking, highest) == cudaSuccess;
        for (cudaEvent_t *event : {&l.fork, &l.sorted, &l.filled, &l.join})
            l.ready = l.ready && cudaEventCreateWithFlags(event, cudaEventDisableTiming) == cudaSuccess;
        if (!l.ready) (void)cudaGetLastError();
    }
    bool free = l.ready;
    if (free && l.user != user) {
        const cudaError_t e = cudaEventQuery(l.join);
        free = e == cudaSuccess;
        if (!free) (void)cudaGetLastError();
    }
    (void)cudaThreadExchangeStreamCaptureMode(&mode);
    if (free) l.user = user;
    return free ? &l : nullptr;
}

// The work list of more than kSmallTokens tokens.
cudaError_t launch_sort(const EmbedGradArgs &a, const GradWork &w, uint32_t slabs, cudaStream_t stream)
{
    const uint32_t n = uint32_t(a.n);
    const unsigned token_blocks = (n + kThreads - 1) / kThreads;
    const unsigned long_blocks = unsigned(max_long(n) < 296 ? max_long(n) : 296);
    cudaError_t e = cudaMemsetAsync(a.workspace, 0, w.zero_bytes, stream);
    if (e == cudaSuccess) e = launch(rd_embed_count_kernel, token_blocks, kThreads, stream, a.ids, a.wide_ids, a.first_row, a.rows, n, w.cnt, w.rank);
    if (e == cudaSuccess) e = launch(rd_embed_ranges_kernel, unsigned((a.rows + 1023) / 1024), 1024, stream, w, a.rows, slabs);
    if (e == cudaSuccess) e = launch(rd_embed_place_kernel, token_blocks, kThreads, stream, a.ids, a.wide_ids, a.first_row, a.rows, n, w.start, w.rank, w.arrived);
    if (e == cudaSuccess)
        e = launch(rd_embed_sort_kernel, token_blocks + long_blocks, kThreads, stream, a.ids, a.wide_ids, a.first_row, a.rows, n, w.cnt, w.start, w.arrived, w.list, w.meta,
                   w.long_row, token_blocks);
    return e;
}

// Rows row0 to row1; `alone`: nothing of the call before it has waited for the stream's earlier work.
template <typename O> cudaError_t launch_fill(const EmbedGradArgs &a, size_t row0, size_t row1, const uint32_t *cnt, bool alone)
{
    const size_t row_bytes = a.dim * sizeof(O), pitch = a.table_stride * sizeof(O), rows = row1 - row0;
    const size_t span = pitch == row_bytes || rows == 1 ? rows * row_bytes : 0;
    const size_t blocks = span ? (span + 31) / kFillBytes + 1 : (rows + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffffu) return cudaErrorInvalidConfiguration;
    return launch(rd_embed_fill_kernel, unsigned(blocks), kThreads, a.stream, static_cast<char *>(a.table) + row0 * pitch, span, rows, row_bytes, pitch,
                  cnt ? cnt + row0 : nullptr, alone);
}

// From this size of table on the fork pays: the sort takes some 20 us, a fork and a join a few.
constexpr size_t kForkBytes = size_t(32) << 20;
// Of a larger table this much is filled while the tokens are sorted, whatever rows have tokens.  The rest, without the rows that
// have tokens, is filled beside the sums, on the SMs that are done with them (both kernels on an SM at once, which takes 96 instead of
// 118 registers here, was slower: a slice of 32768 x 2048 fp32 75 us, this 68).  First part of 64, 128, 192 MB: 69.2, 67.8, 68.0 us
// there, 186.6, 186.8, 185.2 for 131072 x 4096 bf16; everything filled first: 76.7 and 201.6.
constexpr size_t kFirstBytes = size_t(192) << 20;

template <typename T, typename O> cudaError_t launch_stream(const EmbedGradArgs &a, const GradWork &w, uint32_t slabs, cudaStream_t on)
{
    static std::atomic<bool> ready[kMaxDevices];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device >= kMaxDevices || !ready[device].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(rd_embed_stream_kernel<T, O>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem);
        // the fill that runs beside this kernel leaves the shared memory to it: an SM divides its memory anew only when it is idle
        // (slice of 32768 x 2048 fp32: 72 us without this, 68 with it)
        if (e == cudaSuccess) e = cudaFuncSetAttribute(rd_embed_fill_kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        if (e != cudaSuccess) return e;
        if (device < kMaxDevices) ready[device].store(true, std::memory_order_release);
    }
    const uint64_t units = uint64_t(max_big(a.n) + max_items(a.n, a.rows)) * slabs, blocks = (units + kStreamThreads / 32 - 1) / (kStreamThreads / 32);
    cudaLaunchConfig_t c{};
    cudaLaunchAttribute pdl = pdl_attribute();
    c.gridDim = dim3(unsigned(blocks < 148 ? blocks : 148));
    c.blockDim = dim3(kStreamThreads);
    c.dynamicSmemBytes = kStreamSmem;
    c.stream = on;
    c.attrs = &pdl;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, rd_embed_stream_kernel<T, O>, static_cast<const T *>(a.grad), a.grad_stride, static_cast<O *>(a.table), a.table_stride, uint32_t(a.dim), slabs,
                              a.scale, a.accumulate, w);
}

template <typename T, typename O, int V, bool ELEMENTS> cudaError_t launch_grad(const EmbedGradArgs &a)
{
    const GradWork w = layout(a.workspace, a.rows, a.dim, a.n);
    const uint32_t n = uint32_t(a.n);
    const bool stream = !ELEMENTS && a.dim * sizeof(T) >= kStreamBytes;
    const uint32_t vecs = uint32_t((a.dim + V - 1) / V), lanes = lanes_for(vecs);
    const uint32_t slabs = stream ? uint32_t((a.dim * sizeof(T) + kSlab - 1) / kSlab) : (vecs + lanes - 1) / lanes;
    if (n == 0) return a.accumulate ? cudaSuccess : launch_fill<O>(a, 0, a.rows, nullptr, true);
    cudaError_t e = cudaSuccess;
    if (n <= kSmallTokens) {
        e = launch(rd_embed_rank_kernel, (n + 31) / 32, 1024, a.stream, a.ids, a.wide_ids, a.first_row, a.rows, n, w, slabs);
        if (e == cudaSuccess && !a.accumulate) e = launch_fill<O>(a, 0, a.rows, nullptr, false);
    } else {
        std::unique_lock<std::mutex> hold(g_lane_mutex, std::defer_lock);
        Lane *lane = nullptr;
        if (!a.accumulate && a.rows * a.dim * sizeof(O) >= kForkBytes) {
            hold.lock();
            lane = lane_for(a.stream);
        }
        if (lane) {
            const size_t pitch = a.table_stride * sizeof(O), first = !stream ? a.rows : kFirstBytes > pitch ? kFirstBytes / pitch : 1;
            const bool split = first < a.rows;
            cudaError_t f = cudaEventRecord(lane->fork, a.stream);
            if (f == cudaSuccess) f = cudaStreamWaitEvent(lane->side, lane->fork, 0);
            if (f != cudaSuccess) return f;
            e = launch_sort(a, w, slabs, lane->side);
            if (e == cudaSuccess && split) e = cudaEventRecord(lane->sorted, lane->side);
            f = launch_fill<O>(a, 0, split ? first : a.rows, nullptr, true);
            if (e == cudaSuccess && f == cudaSuccess && split) {
                f = cudaEventRecord(lane->filled, a.stream);
                if (f == cudaSuccess) f = cudaStreamWaitEvent(lane->side, lane->filled, 0);
                if (f == cudaSuccess) e = launch_stream<T, O>(a, w, slabs, lane->side);
                if (f == cudaSuccess) f = cudaStreamWaitEvent(a.stream, lane->sorted, 0);
                if (f == cudaSuccess) f = launch_fill<O>(a, first, a.rows, w.cnt, false);
            }
            // joined whatever became of the launches: the caller's stream owns the workspace
            const cudaError_t r = cudaEventRecord(lane->join, lane->side), j = r == cudaSuccess ? cudaStreamWaitEvent(a.stream, lane->join, 0) : r;
            e = e != cudaSuccess ? e : f != cudaSuccess ? f : j;
            if (e != cudaSuccess || split) return e;
        } else {
            e = launch_sort(a, w, slabs, a.stream);
            if (e == cudaSuccess && !a.accumulate) e = launch_fill<O>(a, 0, a.rows, nullptr, false);
        }
    }
    if (e != cudaSuccess) return e;
    if (stream) return launch_stream<T, O>(a, w, slabs, a.stream);
    const uint64_t units = uint64_t(max_big(n) + max_items(n, a.rows)) * slabs, blocks = (units + kThreads / lanes - 1) / (kThreads / lanes);
    return launch(rd_embed_sum_kernel<T, O, V, ELEMENTS>, unsigned(blocks < kSumBlocks ? blocks : kSumBlocks), kThreads, a.stream, static_cast<const T *>(a.grad), a.grad_stride,
                  static_cast<O *>(a.table), a.table_stride, uint32_t(a.dim), lanes, slabs, a.scale, a.accumulate, w);
}

// Vectors of 16 bytes of the gradient's rows when both matrices' rows are made of such, else single elements.
template <typename T, typename O> cudaError_t pick_grad(const EmbedGradArgs &a)
{
    constexpr int V = 16 / sizeof(T);
    const bool wide = vector_rows(a.grad, a.grad_stride, a.dim, sizeof(T), 16) && vector_rows(a.table, a.table_stride, a.dim, sizeof(O), V * sizeof(O));
    return wide ? launch_grad<T, O, V, false>(a) : launch_grad<T, O, 8, true>(a);
}

// Vectors of 32 or 16 bytes when both matrices' rows begin and end on such boundaries (16384 rows of 8 KB, B200: 35 us with 32-byte
// accesses, 39 with 16-byte ones), else single elements.
template <typename T> cudaError_t pick_embed(const EmbedArgs &a)
{
    constexpr int V = 16 / sizeof(T);
    auto fits = [&](size_t to) {
        return vector_rows(a.table, a.table_stride, a.dim, sizeof(T), to) && vector_rows(a.out, a.out_stride, a.dim, sizeof(T), to);
    };
    return fits(32) ? launch_embed<T, 2 * V>(a) : fits(16) ? launch_embed<T, V>(a) : launch_elements<T>(a);
}

}  // namespace

cudaError_t embed_forward(const EmbedArgs &a)
{
    return a.dtype == RD_FP32 ? pick_embed<float>(a) : a.dtype == RD_BF16 ? pick_embed<__nv_bfloat16>(a) : pick_embed<__half>(a);
}

size_t embed_backward_workspace(size_t rows, size_t dim, size_t n) { return layout(nullptr, rows, dim, n).bytes; }

cudaError_t embed_status(int *status)
{
    cudaError_t e = cudaMemcpyFromSymbol(status, g_embed_status, sizeof(int));
    const int zero = 0;
    return e == cudaSuccess && *status ? cudaMemcpyToSymbol(g_embed_status, &zero, sizeof(int)) : e;
}

cudaError_t embed_backward(const EmbedGradArgs &a)
{
    if (a.dtype == RD_FP32) return pick_grad<float, float>(a);
    if (a.dtype == RD_BF16) return a.table_dtype == RD_FP32 ? pick_grad<__nv_bfloat16, float>(a) : pick_grad<__nv_bfloat16, __nv_bfloat16>(a);
    return a.table_dtype == RD_FP32 ? pick_grad<__half, float>(a) : pick_grad<__half, __half>(a);
}

}  // namespace rd
