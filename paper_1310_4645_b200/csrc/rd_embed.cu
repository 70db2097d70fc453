// sm_100a kernels of the embedding lookup and of its gradient.
//
// Lookup:    out[i] = scale * table[ids[i] - first_row], a row of zeros when that row is not in the table.
// Gradient:  g[v] = (accumulate ? g[v] : 0) + scale * sum over the tokens i with ids[i] - first_row = v of grad[i].
//
// Both only move data, so both are bound by HBM: the lookup reads and writes n rows, the gradient reads n rows and writes
// the whole table (the rows no token has get zeros in the same pass).  Sums are fp32 and rounded once at the end.
//
// Gradient.  Tokens are grouped by row, so that every row of the table is written once, by one owner, without
// floating-point atomics: the order of the additions, hence every bit of the result, depends on the ids alone.
//   count    cnt[v] = number of tokens of row v; integer atomics, one per distinct row and warp
//   place    every row with tokens gets a range of the token list (where in the list does not matter), in list order
//            of arrival, which does depend on timing ...
//   sort     ... and is put in ascending order here: each token looks up how many of its row's tokens come before it.
//            Rows with more than kChunk tokens go through a bitmap of token positions in shared memory instead.
//   sum      one group of threads per row adds its tokens' gradients in ascending order.  Rows with more than kChunk
//            tokens are cut into chunks of kChunk, summed side by side into fp32 partial rows,
//   join     which are added in ascending order.
#include "rd_vocab.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "rd.h"
#include "rd_launch.h"

namespace rd {

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kChunk = 64;         // tokens one thread group adds up by itself

template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float widen<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }

// V consecutive elements, moved as one access of up to 16 bytes (two for fp32 results of 16-bit vectors).
template <typename T, int V> struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Vec { T v[V]; };

template <typename T, int V> __device__ __forceinline__ Vec<T, V> load(const T *p) { return *reinterpret_cast<const Vec<T, V> *>(p); }
template <typename T, int V> __device__ __forceinline__ void store(T *p, const Vec<T, V> &x) { *reinterpret_cast<Vec<T, V> *>(p) = x; }

// The table row of token i, or a negative number when the table does not hold it.
__device__ __forceinline__ long long row_of(const void *ids, bool wide, size_t i, long long first, size_t rows)
{
    const long long id = wide ? static_cast<const long long *>(ids)[i] : static_cast<const int *>(ids)[i];
    if (id < first) return -1;                   // first >= 0: negative ids too
    return id - first < static_cast<long long>(rows) ? id - first : -1;
}

constexpr int kGatherUnroll = 4;

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

bool vector_rows(const void *p, size_t stride, size_t dim, size_t esize)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * esize % 16 == 0 && dim * esize % 16 == 0;
}

// ---------------------------------------------------------------------------------------------------- gradient

struct GradMeta {
    uint32_t list_used;       // entries of the token list handed out to rows
    uint32_t n_long;          // rows with more than kChunk tokens
    uint32_t n_chunks;        // their chunks
    uint32_t pad;
};

struct GradWork {             // the workspace's parts
    GradMeta *meta;
    uint32_t *cnt;            // rows
    uint32_t *start;          // rows: where the row's tokens begin in the list
    uint32_t *rank;           // n: arrival number of the token within its row
    uint32_t *arrived;        // n: token list, in order of arrival within a row
    uint32_t *list;           // n: token list, ascending within a row
    uint32_t *long_row;       // rows with more than kChunk tokens
    uint32_t *long_chunk;     // their first chunk
    uint32_t *chunk_row;      // per chunk: index into long_row
    float *partial;           // per chunk: dim fp32 values
    size_t bytes, zero_bytes;
};

size_t max_long(size_t n) { return n / (kChunk + 1); }
size_t max_chunks(size_t n) { return n / kChunk + max_long(n); }

GradWork layout(void *workspace, size_t rows, size_t dim, size_t n)
{
    GradWork w;
    size_t at = 0;
    char *base = static_cast<char *>(workspace);
    auto take = [&](size_t bytes) {
        char *p = base + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    w.meta = reinterpret_cast<GradMeta *>(take(sizeof(GradMeta)));
    w.cnt = reinterpret_cast<uint32_t *>(take(rows * 4));
    w.zero_bytes = at;
    w.start = reinterpret_cast<uint32_t *>(take(rows * 4));
    w.rank = reinterpret_cast<uint32_t *>(take(n * 4));
    w.arrived = reinterpret_cast<uint32_t *>(take(n * 4));
    w.list = reinterpret_cast<uint32_t *>(take(n * 4));
    w.long_row = reinterpret_cast<uint32_t *>(take(max_long(n) * 4));
    w.long_chunk = reinterpret_cast<uint32_t *>(take(max_long(n) * 4));
    w.chunk_row = reinterpret_cast<uint32_t *>(take(max_chunks(n) * 4));
    w.partial = reinterpret_cast<float *>(take(max_chunks(n) * ((dim + 3) / 4 * 4) * 4));
    w.bytes = at;
    return w;
}

__global__ void __launch_bounds__(kThreads) rd_embed_count_kernel(const void *__restrict__ ids, bool wide, long long first, size_t rows, uint32_t n,
                                                                  uint32_t *__restrict__ cnt, uint32_t *__restrict__ rank)
{
    pdl_start();
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

// Hands every row a range of the token list: the ranges of a thread block's rows follow each other.
__global__ void __launch_bounds__(1024) rd_embed_ranges_kernel(const uint32_t *__restrict__ cnt, uint32_t *__restrict__ start, size_t rows, GradMeta *meta,
                                                               uint32_t *__restrict__ long_row, uint32_t *__restrict__ long_chunk, uint32_t *__restrict__ chunk_row)
{
    pdl_start();
    __shared__ uint32_t warp_sum[32];
    __shared__ uint32_t block_base;
    const size_t v = size_t(blockIdx.x) * 1024 + threadIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t c = v < rows ? cnt[v] : 0;
    uint32_t incl = c;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        uint32_t s = warp_sum[lane];
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += o;
        }
        warp_sum[lane] = s;
        if (lane == 31) block_base = s ? atomicAdd(&meta->list_used, s) : 0;
    }
    __syncthreads();
    if (v >= rows) return;
    start[v] = block_base + (warp ? warp_sum[warp - 1] : 0) + incl - c;
    if (c > kChunk) {
        const uint32_t k = atomicAdd(&meta->n_long, 1u);
        const uint32_t chunks = (c + kChunk - 1) / kChunk;
        const uint32_t b = atomicAdd(&meta->n_chunks, chunks);
        long_row[k] = uint32_t(v);
        long_chunk[k] = b;
        for (uint32_t j = 0; j < chunks; j++) chunk_row[b + j] = k;
    }
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

// Sum over list[0..c) of the V values at column j, in list order; four rows in flight.
template <typename T, int V>
__device__ __forceinline__ void add_rows(const T *__restrict__ grad, size_t stride, size_t col, const uint32_t *__restrict__ list, uint32_t c, float (&acc)[V])
{
#pragma unroll
    for (int k = 0; k < V; k++) acc[k] = 0.0f;
    uint32_t t = 0;
    for (; t + 4 <= c; t += 4) {
        Vec<T, V> x[4];
#pragma unroll
        for (int u = 0; u < 4; u++) x[u] = load<T, V>(grad + size_t(list[t + u]) * stride + col);
#pragma unroll
        for (int u = 0; u < 4; u++)
#pragma unroll
            for (int k = 0; k < V; k++) acc[k] += widen<T>(x[u].v[k]);
    }
    for (; t < c; t++) {
        const Vec<T, V> x = load<T, V>(grad + size_t(list[t]) * stride + col);
#pragma unroll
        for (int k = 0; k < V; k++) acc[k] += widen<T>(x.v[k]);
    }
}

template <typename O, int V>
__device__ __forceinline__ void write_row(O *p, const float (&acc)[V], float scale, bool accumulate)
{
    Vec<O, V> y;
    if (accumulate) {
        const Vec<O, V> old = load<O, V>(p);
#pragma unroll
        for (int k = 0; k < V; k++) y.v[k] = narrow<O>(fmaf(acc[k], scale, widen<O>(old.v[k])));
    } else {
#pragma unroll
        for (int k = 0; k < V; k++) y.v[k] = narrow<O>(acc[k] * scale);
    }
    store<O, V>(p, y);
}

// `lanes` (a power of two) threads share a row; thread blocks from row_blocks on take chunks of rows with many tokens.
template <typename T, typename O, int V>
__global__ void __launch_bounds__(kThreads) rd_embed_sum_kernel(const T *__restrict__ grad, size_t grad_stride, O *__restrict__ table, size_t table_stride, size_t rows,
                                                                uint32_t vecs, uint32_t lanes, float scale, bool accumulate, GradWork w, uint32_t row_blocks)
{
    pdl_start();
    const uint32_t per_block = kThreads / lanes, lane = threadIdx.x % lanes, group = threadIdx.x / lanes;
    if (blockIdx.x < row_blocks) {
        const size_t v = size_t(blockIdx.x) * per_block + group;
        if (v >= rows) return;
        const uint32_t c = w.cnt[v];
        if (c > kChunk || (accumulate && c == 0)) return;
        const uint32_t *list = c ? w.list + w.start[v] : w.list;
        for (uint32_t j = lane; j < vecs; j += lanes) {
            float acc[V];
            add_rows<T, V>(grad, grad_stride, size_t(j) * V, list, c, acc);
            write_row<O, V>(table + v * table_stride + size_t(j) * V, acc, scale, accumulate);
        }
        return;
    }
    const uint32_t n_chunks = w.meta->n_chunks;
    for (uint32_t q = (blockIdx.x - row_blocks) * per_block + group; q < n_chunks; q += (gridDim.x - row_blocks) * per_block) {
        const uint32_t k = w.chunk_row[q], v = w.long_row[k], part = q - w.long_chunk[k];
        const uint32_t left = w.cnt[v] - part * kChunk, c = left < kChunk ? left : kChunk;
        const uint32_t *list = w.list + w.start[v] + part * kChunk;
        for (uint32_t j = lane; j < vecs; j += lanes) {
            float acc[V];
            add_rows<T, V>(grad, grad_stride, size_t(j) * V, list, c, acc);
            float *p = w.partial + size_t(q) * ((size_t(vecs) * V + 3) / 4 * 4) + size_t(j) * V;
#pragma unroll
            for (int e = 0; e < V; e++) p[e] = acc[e];
        }
    }
}

template <typename O>
__global__ void __launch_bounds__(kThreads) rd_embed_join_kernel(O *__restrict__ table, size_t table_stride, uint32_t dim, float scale, bool accumulate, GradWork w)
{
    pdl_start();
    const uint32_t n_long = w.meta->n_long;
    const size_t stride = (size_t(dim) + 3) / 4 * 4;
    const uint32_t slabs = (dim + kThreads - 1) / kThreads;
    for (uint64_t u = blockIdx.x; u < uint64_t(n_long) * slabs; u += gridDim.x) {
        const uint32_t q = uint32_t(u / slabs), j = uint32_t(u % slabs) * kThreads + threadIdx.x;
        if (j >= dim) continue;
        const uint32_t v = w.long_row[q], chunks = (w.cnt[v] + kChunk - 1) / kChunk;
        const float *p = w.partial + size_t(w.long_chunk[q]) * stride + j;
        float acc[1] = {0.0f};
        uint32_t k = 0;
        for (; k + 8 <= chunks; k += 8) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; e++) x[e] = p[size_t(k + e) * stride];
#pragma unroll
            for (int e = 0; e < 8; e++) acc[0] += x[e];
        }
        for (; k < chunks; k++) acc[0] += p[size_t(k) * stride];
        write_row<O, 1>(table + size_t(v) * table_stride + j, acc, scale, accumulate);
    }
}

template <typename T, typename O, int V> cudaError_t launch_grad(const EmbedGradArgs &a)
{
    const GradWork w = layout(a.workspace, a.rows, a.dim, a.n);
    const uint32_t n = uint32_t(a.n);
    cudaError_t e = cudaMemsetAsync(a.workspace, 0, w.zero_bytes, a.stream);
    if (e != cudaSuccess) return e;
    const unsigned token_blocks = (n + kThreads - 1) / kThreads;
    const unsigned long_blocks = unsigned(max_long(n) < 296 ? max_long(n) : 296);
    if (n) {
        e = launch(rd_embed_count_kernel, token_blocks, kThreads, a.stream, a.ids, a.wide_ids, a.first_row, a.rows, n, w.cnt, w.rank);
        if (e != cudaSuccess) return e;
        e = launch(rd_embed_ranges_kernel, unsigned((a.rows + 1023) / 1024), 1024, a.stream, w.cnt, w.start, a.rows, w.meta, w.long_row, w.long_chunk, w.chunk_row);
        if (e != cudaSuccess) return e;
        e = launch(rd_embed_place_kernel, token_blocks, kThreads, a.stream, a.ids, a.wide_ids, a.first_row, a.rows, n, w.start, w.rank, w.arrived);
        if (e != cudaSuccess) return e;
        e = launch(rd_embed_sort_kernel, token_blocks + long_blocks, kThreads, a.stream, a.ids, a.wide_ids, a.first_row, a.rows, n, w.cnt, w.start, w.arrived, w.list,
                   w.meta, w.long_row, token_blocks);
        if (e != cudaSuccess) return e;
    }
    const uint32_t vecs = uint32_t(a.dim / V);
    uint32_t lanes = 8;
    while (lanes < uint32_t(kThreads) && lanes < vecs) lanes *= 2;
    const size_t row_blocks = (a.rows + kThreads / lanes - 1) / (kThreads / lanes);
    const size_t chunk_blocks = (max_chunks(n) + kThreads / lanes - 1) / (kThreads / lanes);
    const unsigned extra = unsigned(chunk_blocks < 1184 ? chunk_blocks : 1184);
    if (row_blocks + extra > 0x7fffffffu) return cudaErrorInvalidConfiguration;
    e = launch(rd_embed_sum_kernel<T, O, V>, unsigned(row_blocks) + extra, kThreads, a.stream, static_cast<const T *>(a.grad), a.grad_stride, static_cast<O *>(a.table),
               a.table_stride, a.rows, vecs, lanes, a.scale, a.accumulate, w, uint32_t(row_blocks));
    if (e != cudaSuccess || !long_blocks) return e;
    return launch(rd_embed_join_kernel<O>, 592, kThreads, a.stream, static_cast<O *>(a.table), a.table_stride, uint32_t(a.dim), a.scale, a.accumulate, w);
}

template <typename T, typename O, int V> cudaError_t pick_grad(const EmbedGradArgs &a)
{
    // whole vectors when the gradient's and the table's rows begin and end on 16-byte boundaries
    if (vector_rows(a.grad, a.grad_stride, a.dim, sizeof(T)) && vector_rows(a.table, a.table_stride, a.dim, sizeof(O)) && a.dim % V == 0) return launch_grad<T, O, V>(a);
    return launch_grad<T, O, 1>(a);
}

}  // namespace

cudaError_t embed_forward(const EmbedArgs &a)
{
    const size_t esize = a.dtype == RD_FP32 ? 4 : 2;
    const bool wide = vector_rows(a.table, a.table_stride, a.dim, esize) && vector_rows(a.out, a.out_stride, a.dim, esize);
    if (a.dtype == RD_FP32) return wide ? launch_embed<float, 4>(a) : launch_embed<float, 1>(a);
    if (a.dtype == RD_BF16) return wide ? launch_embed<__nv_bfloat16, 8>(a) : launch_embed<__nv_bfloat16, 1>(a);
    return wide ? launch_embed<__half, 8>(a) : launch_embed<__half, 1>(a);
}

size_t embed_backward_workspace(size_t rows, size_t dim, size_t n) { return layout(nullptr, rows, dim, n).bytes; }

cudaError_t embed_backward(const EmbedGradArgs &a)
{
    if (a.dtype == RD_FP32) return pick_grad<float, float, 4>(a);
    if (a.dtype == RD_BF16) return a.table_dtype == RD_FP32 ? pick_grad<__nv_bfloat16, float, 8>(a) : pick_grad<__nv_bfloat16, __nv_bfloat16, 8>(a);
    return a.table_dtype == RD_FP32 ? pick_grad<__half, float, 8>(a) : pick_grad<__half, __half, 8>(a);
}

}  // namespace rd
