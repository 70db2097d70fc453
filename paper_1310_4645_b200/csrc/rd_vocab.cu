// sm_100a kernels of softmax cross entropy over a large vocabulary and of its gradient, without the logits in memory.
//
//   x_v  = scale * h . w_v                 for the rows w_v of the weight that the call holds
//   lse  = log sum_v exp(x_v),  target = x_label,  loss = lse - target + z * lse^2
//   dx_v = g * ((1 + 2 z lse) exp(x_v - lse) - [v = label]),   dh = scale * sum_v dx_v w_v,   dw_v = scale * sum_tokens dx_v h
//
// Tokens with a negative label count for nothing: a first kernel packs the hidden rows of the others one after another, in
// order, so that ignored rows cost no products and nothing they hold (infinities, NaN) can reach a sum.  Everything after it
// works on the packed rows; how many there are is known on the device only.  Up to 128 tokens are one tile anyway and are taken as
// they lie ("direct"): what ignored rows give is never used, and for dw they are copied, with zeros in their place, beside the
// first product.
//
// Loss.  One matrix product of n x rows x dim whose epilogue keeps, per token and 128 entries of the vocabulary, the maximum and the
// sum of exponentials instead of the logits, and picks out the label's logit; a small kernel joins them.
// Gradient.  In pieces of the vocabulary: the product once more, its epilogue turns logits into dx (16 bits, one rounding:
// the operand type of the products that follow; fp16 dx is scaled by a power of two so that the largest factor g comes near
// the top of the type's range), then both products of the piece in one launch, dw complete, dh added up in fp32 over the pieces.
//
// All three products run on one kernel (tcgen05): a thread block, or a pair of them, computes tiles of 128 x 256 (256 x 256) with
// the accumulators in tensor memory, two sets, so that one is read while the next is computed; operands come in by TMA into a ring
// of stages of 64 summed indices; one warp per operand issues the copies, one the products, eight take the results.
// What bounds it (B200): many tokens, the tensor cores (2048 tokens x 18944 x 4096: 276400 active cycles an SM, 262144 of them
// products) at the clock that the board's power limit leaves, 1.25 to 1.45 GHz: 8192 tokens x 131072 x 4096 loss 6.1 ms = 1.44
// PFLOP/s, gradient 19.4 to 20.5 ms = 1.29 to 1.36.  Few tokens, the memory: 128 tokens x 131072 x 4096 gradient 0.66 ms for 3.2 GB.
// Rows of at most some 256 values, the exponentials: 8192 tokens x 131072 loss 0.54 ms at dim 64 and 128, 0.6 at 256, 0.8 to 0.9 at 512.
#include "rd_vocab.h"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "rd.h"
#include "rd_launch.h"
#include "rd_mma.h"
#include "rd_ptx.h"
#include "rd_ring.h"

namespace rd {

namespace {

constexpr int kPackThreads = 256;
constexpr int kCountTile = 256;           // tokens per thread block of the counting kernel
constexpr size_t kCountFrom = 4097;       // from this many tokens on they are counted by a kernel of their own
constexpr int kRowPad = 256;              // room for packed rows is a multiple of this
constexpr int kZeroPad = 64;              // gradient: zero rows up to a multiple of this, one step of a sum over tokens
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Meta {
    uint32_t m;               // packed rows
    float boost, unboost;     // power of two that dx is multiplied by, and its inverse
    uint32_t pad;
};
struct TileCount {
    uint32_t n;               // tokens of the tile that count
    float most;               // largest finite |factor of dx| among them
};

__device__ __forceinline__ long long label_of(const void *labels, bool wide, size_t i)
{
    return wide ? static_cast<const long long *>(labels)[i] : static_cast<const int *>(labels)[i];
}

struct PackParams {
    const uint16_t *hidden;
    const void *labels;
    size_t hidden_stride, n, rows;
    uint32_t dim, packed_stride;
    long long first;
    bool wide_labels, copy16;
    float scale, z;
    uint16_t *packed;
    int *index, *label;       // per packed row: the token, its label's row in this weight or -1
    const TileCount *tiles;
    Meta *meta;
    // loss
    float *loss, *lse_out, *target;
    // gradient
    const float *lse, *grad_loss;
    size_t grad_loss_stride;
    float *gp, *gt, *lse2;    // per packed row: factor of the probability, of the label's one, lse * log2(e)
    uint16_t *grad_hidden;
    size_t grad_hidden_stride;
    bool gradient, fp16;
};

template <typename P> __device__ __forceinline__ void factors(const P &p, size_t i, float &gp, float &gt)
{
    const float g = p.grad_loss[i * p.grad_loss_stride] * p.scale;
    gt = g;
    gp = p.z != 0.0f ? fmaf(2.0f * p.z * p.lse[i], g, g) : g;
}

// The largest finite factor of dx that token i brings (fp16 only: it decides the power of two).
template <typename P> __device__ __forceinline__ float largest_factor(const P &p, size_t i)
{
    float gp, gt, most = 0.0f;
    factors(p, i, gp, gt);
    if (isfinite(gp)) most = fabsf(gp);
    if (isfinite(gt)) most = fmaxf(most, fabsf(gt));
    return most;
}

__global__ void __launch_bounds__(kCountTile) rd_vocab_count_kernel(PackParams p, TileCount *tiles)
{
    __shared__ float warp_most[kCountTile / 32];
    pdl_wait_first();
    const size_t i = size_t(blockIdx.x) * kCountTile + threadIdx.x;
    const bool counts = i < p.n && label_of(p.labels, p.wide_labels, i) >= 0;
    float most = p.gradient && p.fp16 && counts ? largest_factor(p, i) : 0.0f;
#pragma unroll
    for (int d = 16; d; d /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    if ((threadIdx.x & 31) == 0) warp_most[threadIdx.x >> 5] = most;
    const int n = __syncthreads_count(counts);
    if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 1; k < kCountTile / 32; k++) most = fmaxf(most, warp_most[k]);
        tiles[blockIdx.x] = TileCount{uint32_t(n), most};
    }
}

// fp16: the power of two that takes the largest factor to [2^13, 2^14); probabilities down to 2^-27 of it stay normal numbers.
__device__ __forceinline__ float boost_for(float most)
{
    if (!(most > 0.0f)) return 1.0f;
    int e;
    frexpf(most, &e);
    e = 14 - e;
    return ldexpf(1.0f, e > 100 ? 100 : e < -100 ? -100 : e);
}

// `threads` threads copy a row; the copy's row has room for a multiple of 8 elements, and zeros there.
__device__ __forceinline__ void copy_row(uint16_t *dst, const uint16_t *src, uint32_t n, uint32_t padded, bool wide, int t, int threads)
{
    if (wide) {
        const uint4 *s = reinterpret_cast<const uint4 *>(src);
        uint4 *d = reinterpret_cast<uint4 *>(dst);
#pragma unroll 8
        for (uint32_t j = t; j < n / 8; j += threads) d[j] = s[j];
    } else {
#pragma unroll 4
        for (uint32_t j = t; j < padded; j += threads) dst[j] = j < n ? src[j] : uint16_t(0);
    }
}

// Thread blocks below pack_blocks: R tokens each, kPackThreads / R threads copy a row.  Every block finds out for itself how many
// tokens before its own count, from the counting kernel's tiles or, where there are none (n_tiles = 0), from the labels.
// The other blocks (gradient): the zero rows behind the packed ones.
template <int R> __global__ void __launch_bounds__(kPackThreads) rd_vocab_pack_kernel(PackParams p, uint32_t pack_blocks, uint32_t n_tiles)
{
    constexpr int kWarps = kPackThreads / 32, kRowThreads = kPackThreads / R;
    __shared__ uint32_t sums[2][kWarps];
    __shared__ float mosts[kWarps];
    __shared__ uint32_t mask_of_block;
    pdl_wait_first();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool packs = blockIdx.x < pack_blocks, first = blockIdx.x == 0;
    const size_t base = packs ? size_t(blockIdx.x) * R : p.n;          // first token of the block
    uint32_t before = 0, all = 0;                                      // tokens that count, before the block and in all
    float most = 0.0f;
    if (n_tiles) {
        const uint32_t own_tile = uint32_t(base / kCountTile);
        for (uint32_t t = threadIdx.x; t < n_tiles; t += kPackThreads) {
            const TileCount c = p.tiles[t];
            all += c.n;
            if (t < own_tile) before += c.n;
            most = fmaxf(most, c.most);
        }
        const size_t i = size_t(own_tile) * kCountTile + threadIdx.x;
        if (i < base && i < p.n && label_of(p.labels, p.wide_labels, i) >= 0) before++;
    } else {
#pragma unroll 8
        for (uint32_t i = threadIdx.x; i < uint32_t(p.n); i += kPackThreads) {
            const uint32_t counts = label_of(p.labels, p.wide_labels, i) >= 0;
            all += counts;
            before += i < base ? counts : 0;
        }
        if (p.gradient && p.fp16 && first)
            for (uint32_t i = threadIdx.x; i < uint32_t(p.n); i += kPackThreads)
                if (label_of(p.labels, p.wide_labels, i) >= 0) most = fmaxf(most, largest_factor(p, i));
    }
#pragma unroll
    for (int d = 16; d; d /= 2) {
        before += __shfl_xor_sync(0xffffffffu, before, d);
        all += __shfl_xor_sync(0xffffffffu, all, d);
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    }
    if (lane == 0) {
        sums[0][warp] = before;
        sums[1][warp] = all;
        mosts[warp] = most;
    }
    if (warp == 0 && packs) {
        const bool counts = lane < R && base + lane < p.n && label_of(p.labels, p.wide_labels, base + lane) >= 0;
        const uint32_t b = __ballot_sync(0xffffffffu, counts);
        if (lane == 0) mask_of_block = b;
    }
    __syncthreads();
    before = all = 0;
    most = 0.0f;
#pragma unroll
    for (int k = 0; k < kWarps; k++) {
        before += sums[0][k];
        all += sums[1][k];
        most = fmaxf(most, mosts[k]);
    }
    if (first && threadIdx.x == 0) {
        const float boost = p.fp16 ? boost_for(most) : 1.0f;
        *p.meta = Meta{all, boost, 1.0f / boost, 0};
    }
    const int row = threadIdx.x / kRowThreads, t = threadIdx.x % kRowThreads;
    if (!packs) {
        const size_t r = size_t(all) + (blockIdx.x - pack_blocks) * R + row;
        if (r >= (size_t(all) + kZeroPad - 1) / kZeroPad * kZeroPad) return;
        uint4 *dst = reinterpret_cast<uint4 *>(p.packed + r * p.packed_stride);
        for (uint32_t j = t; j < p.packed_stride / 8; j += kRowThreads) dst[j] = make_uint4(0, 0, 0, 0);
        return;
    }
    const size_t i = base + row;
    if (i >= p.n) return;
    const uint32_t mask = mask_of_block;
    if (!(mask >> row & 1)) {
        if (p.gradient) {
            if (p.grad_hidden)
                for (uint32_t j = t; j < p.dim; j += kRowThreads) p.grad_hidden[i * p.grad_hidden_stride + j] = 0;
        } else if (t == 0) {
            if (p.loss) p.loss[i] = 0.0f;
            if (p.lse_out) p.lse_out[i] = 0.0f;
            if (p.target) p.target[i] = 0.0f;
        }
        return;
    }
    const size_t r = size_t(before) + __popc(mask & ((1u << row) - 1));
    copy_row(p.packed + r * p.packed_stride, p.hidden + i * p.hidden_stride, p.dim, p.packed_stride, p.copy16, t, kRowThreads);
    if (t == 0) {
        const long long l = label_of(p.labels, p.wide_labels, i);
        p.index[r] = int(i);
        p.label[r] = l >= p.first && l - p.first < static_cast<long long>(p.rows) ? int(l - p.first) : -1;
        if (p.gradient) {
            float gp, gt;
            factors(p, i, gp, gt);
            p.gp[r] = gp;
            p.gt[r] = gt;
            p.lse2[r] = p.lse[i] * kLog2e;
        }
    }
}

// Copies a weight whose rows TMA cannot address (unaligned base or stride) to rows that it can.
__global__ void __launch_bounds__(kPackThreads) rd_vocab_align_kernel(uint16_t *dst, uint32_t dst_stride, const uint16_t *src, size_t src_stride, size_t rows, uint32_t dim)
{
    pdl_start();
    for (size_t r = size_t(blockIdx.x) * (kPackThreads / 32) + (threadIdx.x >> 5); r < rows; r += size_t(gridDim.x) * (kPackThreads / 32))
        copy_row(dst + r * dst_stride, src + r * src_stride, dim, dst_stride, false, threadIdx.x & 31, 32);
}

// ------------------------------------------------------------------------------------------------ the products

constexpr int kMmaThreads = 128 + 32 * kEpilogueWarps;

// Where a row of the products comes from: packed rows have their tokens and labels in lists, direct ones are the tokens themselves.
struct Rows {
    const int *index, *label;
    const void *labels;
    long long first;
    size_t rows;
    bool direct, wide;
    __device__ __forceinline__ size_t token(uint32_t row) const { return direct ? row : size_t(index[row]); }
    __device__ __forceinline__ bool counts(uint32_t row) const { return !direct || label_of(labels, wide, row) >= 0; }
    // the label's row in this weight, -1 where it has none
    __device__ __forceinline__ int label_row(uint32_t row, bool &counts) const
    {
        counts = true;
        if (!direct) return label[row];
        const long long l = label_of(labels, wide, row);
        counts = l >= 0;
        return l >= first && l - first < static_cast<long long>(rows) ? int(l - first) : -1;
    }
};

// Direct rows of the gradient: what the packing kernel would have worked out.
struct Direct {
    uint32_t n;
    const uint16_t *hidden;
    size_t hidden_stride;
    uint16_t *packed;         // the copy that dw reads, null where it is not wanted
    uint32_t packed_stride;
    const float *lse, *grad_loss;
    size_t grad_loss_stride;
    float scale, z;
    Meta *meta;
    bool copy16;
};

struct JoinParams {
    const float2 *part;
    const float *packed_target;
    Rows rows;
    const Meta *meta;
    uint32_t n;               // direct rows
    uint32_t row0, rows_most; // the band, as below
    uint32_t parts;
    float z;
    float *loss, *lse, *target;
};

// Joins (maximum, sum) with another; a part whose maximum is infinite has its sum relative to 0.
__device__ __forceinline__ void join_parts(float2 &x, float2 y)
{
    const float most = fmaxf(x.x, y.x), ref = fabsf(most) == INFINITY ? 0.0f : most;
    const float a = fabsf(x.x) == INFINITY ? x.y : x.y * exp2f(x.x - ref), b = fabsf(y.x) == INFINITY ? y.y : y.y * exp2f(y.x - ref);
    x = make_float2(most, a + b);
}
// A row's parts, joined by a warp; the result is lane 0's.
__device__ __forceinline__ float2 join_row(const float2 *part, uint32_t parts, int lane)
{
    float2 x = make_float2(-INFINITY, 0.0f);
    for (uint32_t k = lane; k < parts; k += 256) {
        float2 y[8];
#pragma unroll
        for (int u = 0; u < 8; u++) y[u] = k + 32 * u < parts ? part[k + 32 * u] : make_float2(-INFINITY, 0.0f);
#pragma unroll
        for (int u = 0; u < 8; u++) join_parts(x, y[u]);
    }
#pragma unroll
    for (int d = 16; d; d /= 2) join_parts(x, make_float2(__shfl_down_sync(0xffffffffu, x.x, d), __shfl_down_sync(0xffffffffu, x.y, d)));
    return x;
}
__device__ __forceinline__ void write_row(float2 x, bool counts, float target, float z, size_t i, int lane, float *loss, float *lse_out, float *target_out)
{
    if (lane) return;
    const float ref = fabsf(x.x) == INFINITY ? 0.0f : x.x;
    const float lse = counts ? (ref + log2f(x.y)) * kLn2 : 0.0f;
    // without the penalty an infinite lse is an infinite loss, not 0 * inf
    if (loss) loss[i] = !counts ? 0.0f : z != 0.0f ? lse - target + z * lse * lse : lse - target;
    if (lse_out) lse_out[i] = lse;
    if (target_out) target_out[i] = target;
}

struct alignas(64) MmaParams {
    CUtensorMap a_k;          // rows of the left operand, 64 x a_rows boxes: packed hidden (stats, dlogits), dx (dh)
    CUtensorMap b_k;          // rows of the weight, 64 x 256 boxes (stats, dlogits)
    CUtensorMap a_mn;         // dx as the transposed left operand of dw, 64 x 64 boxes
    CUtensorMap b_mn;         // weight as the transposed right operand of dh
    CUtensorMap b2_mn;        // packed hidden as the transposed right operand of dw
    CUtensorMap dx_out;       // dx, 64 x 32 boxes
    CUtensorMap dh_out;       // dh, 32 x 32 x 1 boxes
    CUtensorMap dw_out;       // grad_weight, 64 x 32 boxes
    const Meta *meta;
    Rows rows;
    Direct direct;            // logits
    const float *gp, *gt, *lse2;
    float2 *part;             // stats: (maximum, sum) in base 2, [row][part]
    float *target;            // stats: the label's logit, per packed row
    uint16_t *dw;             // grad_weight, for rows that TMA cannot address
    uint16_t *gh;             // grad_hidden, where one part of dh is all of it
    size_t dh_stride, dw_stride, gh_stride;
    uint32_t row0, rows_most; // stats: first row of the band of rows that the launch covers, and its room
    uint32_t parts;           // stats: parts per row, two to a tile of 256 columns, one to a smaller one
    uint32_t piece0, piece;   // first row of the piece and its rows
    uint32_t dim;
    uint32_t tile_n;          // logits: columns of a tile, 256, 128 or 64
    uint32_t stages, stage;   // logits: stages of the ring and bytes of one
    uint32_t group;           // token tiles that go over the vocabulary together
    uint32_t splits;          // parts that the sum over the piece is cut into for dh
    uint32_t a_rows;          // rows of a thread block's left operand that are brought in (fewer than 128 for few tokens)
    bool first_piece, want_dh, want_dw, dw_tma;
    bool gh_wide;             // 16-byte rows of grad_hidden
    float scale2;             // scale * log2(e)
    float scale;
};

constexpr uint32_t kTileOverhead = 2;     // what a tile costs besides its products, in steps of the summed index

// One unit of work: an output tile and the range of the summed index that goes into it.
struct Work {
    int product;              // 0 logits, 1 dh, 2 dw
    uint32_t m0, n0, k0, kblocks, split;
};

// Which units of work a group of thread blocks (one or a pair, number c of g) gets: next() until it says no.
// Logits: bands of p.group token tiles, within a band all token tiles of a vocabulary tile one after the other.
// Gradients: the units of dh first, dealt out in turn; their number need not divide by g, so some groups get one more of them,
// and that many fewer of dw's tiles, by the number of steps of the summed index.  Few tokens (single blocks): every other block takes
// dw first, so that dh's reading of the weight and dw's writing overlap (64 tokens x 10000 x 2048, B200: 38 us all with dh first,
// 33 so).
template <int KIND, int CG> struct Plan {
    static constexpr uint32_t kTileM = Shape<KIND, CG>::tile_m;
    const MmaParams &p;
    Cursor at;
    uint32_t c, g, tiles_m;
    uint32_t tiles_n, band, k_dim;                             // logits
    uint32_t left, phase, turn, split, dh_n, k_per_split, k_piece, dh_mine, dh_more;    // gradients: units left in the phase (0 dh, 1 dw, 2 dw's rest)
    uint32_t dw_tiles, k_tokens, dw_even;
    bool dw_first;

    __device__ __forceinline__ Plan(const MmaParams &params, uint32_t m) : p(params), c(blockIdx.x / CG), g(gridDim.x / CG)
    {
        if (KIND == kStats) m = m > p.row0 ? min(m - p.row0, p.rows_most) : 0;
        tiles_m = (m + kTileM - 1) / kTileM;
        if (KIND != kGrads) {
            tiles_n = (p.piece + p.tile_n - 1) / p.tile_n;
            k_dim = (p.dim + kTileK - 1) / kTileK;
            band = 0;
            if (tiles_m) at.set(c, g, min(p.group, tiles_m));
        } else {
            dh_n = (p.dim + kTileN - 1) / kTileN;
            k_piece = (p.piece + kTileK - 1) / kTileK;
            k_per_split = (k_piece + p.splits - 1) / p.splits;
            k_tokens = (m + kTileK - 1) / kTileK;
            dw_tiles = p.want_dw ? (p.piece + kTileM - 1) / kTileM * dh_n : 0;
            const uint32_t dh_units = p.want_dh ? tiles_m * dh_n * p.splits : 0;
            dh_more = dh_units % g;                            // groups with one more unit of dh
            // a unit of dh is worth this many tiles of dw, which the other groups take first
            const uint32_t worth = dh_more ? (2 * (k_per_split + kTileOverhead) + k_tokens) / (2 * (k_tokens + kTileOverhead)) : 0;
            const uint32_t ahead = worth * (g - dh_more);
            dw_even = dw_tiles > ahead ? (dw_tiles - ahead + g - 1) / g : 0;      // turns that every group takes part in
            dh_mine = dh_units / g + (c < dh_more);
            split = 0;
            turn = 0;
            dw_first = CG == 1 && (c & 1);
            enter(dw_first ? 1 : 0);
        }
    }
    // gradients: the first unit of a phase
    __device__ __forceinline__ void enter(uint32_t p)
    {
        phase = p;
        if (p == 0) {
            left = dh_mine;
            at.set(c, g, dh_n);
        } else if (p == 1) {
            left = dw_even;
            at.set(c, g, dh_n);
        } else {
            left = c < dh_more ? 0 : 0xffffffffu;              // until the tiles run out
            at.set(dw_even * g + c - dh_more, g - dh_more, dh_n);
        }
    }
    __device__ __forceinline__ bool next(Work &w)
    {
        if constexpr (KIND != kGrads) {
            if (tiles_m == 0) return false;
            while (at.y >= tiles_n) {                          // on to the next band
                const uint32_t over = (at.y - tiles_n) * at.wide + at.x;
                if (++band * p.group >= tiles_m) {
                    band--;                                    // stay at the end
                    return false;
                }
                at.set(over, g, min(p.group, tiles_m - band * p.group));
            }
            w = Work{0, (KIND == kStats ? p.row0 : 0) + (band * p.group + at.x) * kTileM, at.y * p.tile_n, 0, k_dim, 0};
            at.advance();
            return true;
        } else {
            for (;;) {
                if (left == 0 || (phase != 0 && at.y * dh_n + at.x >= dw_tiles)) {
                    if (++turn == 3) {
                        turn = 2;                              // stay at the end
                        left = 0;
                        return false;
                    }
                    enter(dw_first ? (turn + 1) % 3 : turn);
                    continue;
                }
                break;
            }
            if (phase == 0) {
                while (at.y >= tiles_m) {
                    at.y -= tiles_m;
                    split++;
                }
                const uint32_t k0 = split * k_per_split, k1 = min(k0 + k_per_split, k_piece);
                w = Work{1, at.y * kTileM, at.x * kTileN, k0 * kTileK, k1 > k0 ? k1 - k0 : 0, split};
            } else {
                w = Work{2, at.y * kTileM, at.x * kTileN, 0, k_tokens, 0};
            }
            left--;
            at.advance();
            return true;
        }
    }
};

template <int KIND, bool BF16, int CG>
__global__ void __launch_bounds__(kMmaThreads, 1) rd_vocab_mma_kernel(const __grid_constant__ MmaParams p)
{
    using S = Shape<KIND, CG>;
    const uint32_t stages = KIND == kGrads ? uint32_t(S::stages) : p.stages, stage = KIND == kGrads ? uint32_t(S::stage) : p.stage;
    const uint32_t stage_a = KIND == kGrads ? uint32_t(S::stage_a) : p.a_rows * kTileK * 2;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t smem = (smem_addr(smem_raw) + 1023) & ~1023u;
    const uint32_t boxes = smem + S::ring, bars = boxes + S::boxes;
    // barriers: full[stage], empty[stage], accumulator full[2], empty[2]; then the tensor memory address
    const uint32_t full = bars, empty = bars + 8 * kMostStages, acc_full = bars + 16 * kMostStages, acc_empty = acc_full + 16, tmem_slot = acc_empty + 16;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? blockIdx.x & 1 : 0;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < stages; s++) {
            bar_init(full + 8 * s, 1);
            bar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; b++) {
            bar_init(acc_full + 8 * b, 1);
            bar_init(acc_empty + 8 * b, kEpilogueWarps * CG);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3 && lane == 0) {
        for (const CUtensorMap *map : {&p.a_k, KIND == kGrads ? &p.b_mn : &p.b_k}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
        if (KIND == kGrads)
            for (const CUtensorMap *map : {&p.a_mn, &p.b2_mn}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    if (warp == 2) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tmem_slot) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tmem_slot) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    pair_sync<CG>();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));

    // direct rows: this is the call's first kernel
    const bool direct = KIND != kGrads && CG == 1 && p.rows.direct;
    if (direct) pdl_wait_first();
    else pdl_start();
    const uint32_t m = __shfl_sync(0xffffffffu, direct ? p.direct.n : p.meta->m, 0);
    Plan<KIND, CG> plan(p, m);
    bool dead = false;

    if (warp == 0 || warp == 3) {
        // one warp brings in the left operand, another the right one
        const bool elected = elect_one();
        Turn turn(stages);
        Work w;
        const uint32_t lead = leader_bar<CG>(full);
        while (!dead && plan.next(w)) {
            const uint32_t rows_n = KIND != kGrads ? p.tile_n / CG : uint32_t(S::rows_n);
            const uint32_t m0 = w.m0 + rank * kRowsM, n0 = w.n0 + rank * rows_n;
            const uint32_t bytes = CG * ((w.product == 2 ? S::stage_a : p.a_rows * kTileK * 2) + rows_n * kTileK * 2);
            const CUtensorMap *map_b = w.product == 1 ? &p.b_mn : &p.b2_mn;
            const uint32_t y0 = w.product == 1 ? p.piece0 : 0;
            for (uint32_t k = 0, kk = w.k0; k < w.kblocks; k++, kk += kTileK, turn.advance()) {
                const uint32_t a = smem + turn.s * stage, b = a + stage_a, bar = lead + 8 * turn.s;
                if (!warp_wait(empty + 8 * turn.s, turn.parity ^ 1)) { dead = true; break; }
                if (warp == 0) {
                    if (elected) {
                        // the copies of both thread blocks and both operands count at the first block's barrier
                        if (rank == 0) bar_expect(full + 8 * turn.s, bytes);
                        if (w.product == 2) {
#pragma unroll
                            for (int j = 0; j < kRowsM / 64; j++) tma_load<CG>(a + j * 8192, &p.a_mn, m0 + 64 * j, kk, bar);
                        } else {
                            tma_load<CG>(a, &p.a_k, kk, m0, bar);
                        }
                    }
                } else if (elected) {
                    if (KIND != kGrads) {
                        tma_load<CG>(b, &p.b_k, kk, p.piece0 + n0, bar);
                    } else {
#pragma unroll
                        for (int j = 0; j < S::rows_n / 64; j++) tma_load<CG>(b + j * 8192, map_b, n0 + 64 * j, y0 + kk, bar);
                    }
                }
            }
        }
        // the last stages' arrivals have to land while the barriers still exist
        for (uint32_t s = 0; s < stages && !dead; s++, turn.advance()) dead = !warp_wait(empty + 8 * turn.s, turn.parity ^ 1);
        if (dead) drain();
    } else if (warp == 1) {
        if (rank == 0) {
            const bool elected = elect_one();
            const uint32_t desc = 1u << 4 | (BF16 ? 1u << 7 | 1u << 10 : 0u) | (KIND != kGrads ? p.tile_n : kTileN) / 8 << 17 | uint32_t(S::tile_m / 16) << 24;
            Turn turn(stages);
            uint32_t tile = 0;
            Work w;
            while (!dead && plan.next(w)) {
                if (w.kblocks == 0) continue;            // the epilogue takes zeros
                const uint32_t buf = tile & 1;
                if (!warp_wait(acc_empty + 8 * buf, (tile / 2 & 1) ^ 1)) { dead = true; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const bool ta = w.product == 2, tb = w.product != 0;
                const uint32_t idesc = desc | (ta ? 1u << 15 : 0u) | (tb ? 1u << 16 : 0u);
                const uint32_t step_a = ta ? 2048 >> 4 : 32 >> 4, step_b = tb ? 2048 >> 4 : 32 >> 4;
                const uint32_t acc = tmem + buf * kTileN;
                for (uint32_t k = 0; k < w.kblocks; k++, turn.advance()) {
                    const uint32_t a = smem + turn.s * stage, b = a + stage_a;
                    if (!warp_wait(full + 8 * turn.s, turn.parity)) { dead = true; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = operand(a, ta), db = operand(b, tb);
                    if (elected) {
#pragma unroll
                        for (int j = 0; j < kTileK / 16; j++) mma<CG>(acc, da + j * step_a, db + j * step_b, idesc, k != 0 || j != 0);
                        mma_commit<CG>(empty + 8 * turn.s);
                    }
                }
                if (!dead && elected) mma_commit<CG>(acc_full + 8 * buf);
                tile++;
            }
            if (dead) drain();
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, half = (warp - 4) >> 2;        // rows 32 * quarter.., columns 128 * half.. of the tile
        const uint32_t box = boxes + (warp - 4) * kBox;
        uint32_t tile = 0;
        Work w;
        float boost = 1.0f;
        if (KIND == kDlogits && direct) {
            // what the packing kernel does otherwise: the power of two, and for dw the rows that count, with zeros in the others' place
            // and behind the last one
            const Direct &d = p.direct;
            if (!BF16) {
                float most = 0.0f;
                for (uint32_t i = lane; i < d.n; i += 32)
                    if (p.rows.counts(i)) most = fmaxf(most, largest_factor(d, i));
#pragma unroll
                for (int x = 16; x; x /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
                boost = boost_for(most);
            }
            if (p.first_piece) {
                if (blockIdx.x == 0 && threadIdx.x == 128) *d.meta = Meta{d.n, boost, 1.0f / boost, 0};
                if (d.packed)
                    for (uint32_t r = blockIdx.x * kEpilogueWarps + warp - 4; r < (d.n + kZeroPad - 1) / kZeroPad * kZeroPad; r += gridDim.x * kEpilogueWarps) {
                        const bool counts = r < d.n && p.rows.counts(r);
                        uint16_t *dst = d.packed + size_t(r) * d.packed_stride;
                        if (counts) copy_row(dst, d.hidden + size_t(r) * d.hidden_stride, p.dim, d.packed_stride, d.copy16, lane, 32);
                        else
                            for (uint32_t j = lane; j < d.packed_stride / 8; j += 32) reinterpret_cast<uint4 *>(dst)[j] = make_uint4(0, 0, 0, 0);
                    }
            }
        } else if (KIND == kDlogits) {
            boost = p.meta->boost;
        }
        while (plan.next(w)) {
            const uint32_t row0 = w.m0 + rank * kRowsM + 32 * quarter, row = row0 + lane, col0 = w.n0 + 128 * half;
            const uint32_t buf = tile & 1;
            if (w.kblocks) {
                if (!warp_wait(acc_full + 8 * buf, tile / 2 & 1)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
            const uint32_t acc = tmem + buf * kTileN + 128 * half + (uint32_t(32 * quarter) << 16);
            // the row's numbers (stats and dlogits)
            int label = -1;
            float lse2 = 0.0f, gp = 0.0f, gt = 0.0f;
            bool live = KIND != kGrads && row < m;
            if (live) {
                label = p.rows.label_row(row, live);
                if (KIND == kDlogits && live) {
                    if (direct) {
                        factors(p.direct, row, gp, gt);
                        lse2 = p.direct.lse[row] * kLog2e;
                    } else {
                        lse2 = p.lse2[row];
                        gp = p.gp[row];
                        gt = p.gt[row];
                    }
                    gp *= boost;
                    gt *= boost;
                    label = label < int(p.piece0) ? -1 : label - int(p.piece0);
                }
            }
            // columns of the tile that the vocabulary has; in tiles of fewer than 256 the rest is another tile's
            const uint32_t limit = KIND != kGrads ? min(p.piece, w.n0 + p.tile_n) : 0;
            const float unboost = KIND == kGrads && !BF16 ? p.meta->unboost : 1.0f;      // bf16: always 1, and no multiplication
            // the accumulators are free for the next tile but one as soon as their last columns are in registers
            auto release = [&]() {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive_leader<CG>(acc_empty + 8 * buf);
            };
            if constexpr (KIND == kStats) {
                // The warp's 128 columns at once: one maximum, then the sum.  32768 exponentials per thread block and tile at
                // 16 a cycle are what bounds this, about 2000 cycles of a tile's 512 per 64 of dim.
                uint32_t v[4][32];
#pragma unroll
                for (int c = 0; c < 4; c++) tmem_load(acc + 32 * c, v[c]);
#pragma unroll
                for (int c = 0; c < 4; c++) tmem_wait(v[c]);
                release();
                if (col0 + 128 > limit) {
                    // the lowest value in the columns that the vocabulary does not have
                    const uint32_t lowest = __float_as_uint(p.scale2 >= 0.0f ? -INFINITY : INFINITY);
#pragma unroll
                    for (int c = 0; c < 4; c++)
#pragma unroll
                        for (int j = 0; j < 32; j++)
                            if (col0 + 32 * c + j >= limit) v[c][j] = lowest;
                }
                if (label >= 0 && uint32_t(label) - col0 < 128u && uint32_t(label) < limit) {
#pragma unroll
                    for (int c = 0; c < 4; c++)
#pragma unroll
                        for (int j = 0; j < 32; j++)
                            if (uint32_t(label) == col0 + 32 * c + j) p.target[row] = __uint_as_float(v[c][j]) * p.scale;
                }
                float t[8];
#pragma unroll
                for (int j = 0; j < 8; j++) t[j] = __uint_as_float(v[0][j]);
                if (p.scale2 >= 0.0f) {
#pragma unroll
                    for (int j = 8; j < 128; j++) t[j & 7] = fmaxf(t[j & 7], __uint_as_float(v[j / 32][j % 32]));
#pragma unroll
                    for (int d = 4; d; d /= 2)
#pragma unroll
                        for (int j = 0; j < d; j++) t[j] = fmaxf(t[j], t[j + d]);
                } else {
#pragma unroll
                    for (int j = 8; j < 128; j++) t[j & 7] = fminf(t[j & 7], __uint_as_float(v[j / 32][j % 32]));
#pragma unroll
                    for (int d = 4; d; d /= 2)
#pragma unroll
                        for (int j = 0; j < d; j++) t[j] = fminf(t[j], t[j + d]);
                }
                const float top = t[0] * p.scale2;
                // an infinite maximum must not meet itself in a difference: exp2(inf) and exp2(-inf) are right as they are
                const float ref = fabsf(top) == INFINITY ? 0.0f : top;
                float sum[8] = {};
#pragma unroll
                for (int j = 0; j < 128; j++) sum[j & 7] += exp2_fast(fmaf(__uint_as_float(v[j / 32][j % 32]), p.scale2, -ref));
#pragma unroll
                for (int d = 4; d; d /= 2)
#pragma unroll
                    for (int j = 0; j < d; j++) sum[j] += sum[j + d];
                if (row < min(m, p.row0 + p.rows_most) && col0 < w.n0 + p.tile_n)
                    p.part[size_t(row - p.row0) * p.parts + (p.tile_n == kTileN ? col0 / 128 : w.n0 / p.tile_n)] = make_float2(top, sum[0]);
            } else {
                auto take = [&](int c, uint32_t (&v)[32]) {
                    const uint32_t col = col0 + 32 * c;
                    if constexpr (KIND == kDlogits) {
                        float y[32];
#pragma unroll
                        for (int j = 0; j < 32; j++) {
                            y[j] = exp2_fast(fmaf(__uint_as_float(v[j]), p.scale2, -lse2)) * gp;
                            if (col + j == uint32_t(label)) y[j] -= gt;
                            if (!live || col + j >= limit) y[j] = 0.0f;
                        }
                        box_wait(lane, c & 1);
#pragma unroll
                        for (int q = 0; q < 4; q++)
                            box_put(box, lane, 4 * (c & 1) + q, pack2<BF16>(y[8 * q], y[8 * q + 1]), pack2<BF16>(y[8 * q + 2], y[8 * q + 3]), pack2<BF16>(y[8 * q + 4], y[8 * q + 5]),
                                    pack2<BF16>(y[8 * q + 6], y[8 * q + 7]));
                        if (box_full(lane, c & 1) && col - 32 < w.n0 + p.tile_n) {
                            tma_store(&p.dx_out, box, col - 32, row0);
                            box_sent();
                        }
                    } else {
                        if (w.product == 1 && p.gh) {
                            if (row < m) {
                                uint16_t *dst = p.gh + p.rows.token(row) * p.gh_stride + col;
                                const bool counts = p.rows.counts(row);         // else zeros, whatever the weight holds
#pragma unroll
                                for (int q = 0; q < 4; q++) {
                                    uint32_t o[4];
#pragma unroll
                                    for (int j = 0; j < 4; j++) o[j] = counts ? pack2<BF16>(__uint_as_float(v[8 * q + 2 * j]) * unboost, __uint_as_float(v[8 * q + 2 * j + 1]) * unboost) : 0;
                                    if (p.gh_wide && col + 8 * q + 8 <= p.dim) {
                                        *reinterpret_cast<uint4 *>(dst + 8 * q) = make_uint4(o[0], o[1], o[2], o[3]);
                                    } else {
#pragma unroll
                                        for (int j = 0; j < 8; j++)
                                            if (col + 8 * q + j < p.dim) dst[8 * q + j] = uint16_t(o[j / 2] >> (j & 1 ? 16 : 0));
                                    }
                                }
                            }
                        } else if (w.product == 1) {
                            box_wait(lane, false);
#pragma unroll
                            for (int q = 0; q < 8; q++) box_put(box, lane, q, v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                            if (box_full(lane, true) && col < p.dh_stride && row0 < m) {
                                if (p.first_piece) tma_store(&p.dh_out, box, col, row0, w.split);
                                else tma_add(&p.dh_out, box, col, row0, w.split);
                                box_sent();
                            }
                        } else {
                            box_wait(lane, c & 1);
#pragma unroll
                            for (int q = 0; q < 4; q++) {
                                uint32_t o[4];
#pragma unroll
                                for (int j = 0; j < 4; j++) o[j] = pack2<BF16>(__uint_as_float(v[8 * q + 2 * j]) * unboost, __uint_as_float(v[8 * q + 2 * j + 1]) * unboost);
                                box_put(box, lane, 4 * (c & 1) + q, o[0], o[1], o[2], o[3]);
                            }
                            if (p.dw_tma && box_within(col - 32 * (c & 1), p.dim)) {
                                if (box_full(lane, c & 1) && col - 32 < p.dim && row0 < p.piece) {
                                    tma_store(&p.dw_out, box, col - 32, p.piece0 + row0);
                                    box_sent();
                                }
                            } else if (c & 1) {
                                // rows that TMA cannot address, or whose end it would overwrite: the warp writes them one after the
                                // other, two elements a lane
                                __syncwarp();
                                const uint32_t rows = row0 < p.piece ? min(32u, p.piece - row0) : 0;
                                uint16_t *dst = p.dw + size_t(p.piece0 + row0) * p.dw_stride + (col - 32);
#pragma unroll 4
                                for (uint32_t r = 0; r < rows; r++) {
#pragma unroll
                                    for (int i = 0; i < 2; i++) {
                                        const uint32_t j = lane + 32 * i;
                                        uint16_t x;
                                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(box + r * 128 + (((j / 8) ^ (r & 7)) * 16) + j % 8 * 2) : "memory");
                                        if (col - 32 + j < p.dim) dst[size_t(r) * p.dw_stride + j] = x;
                                    }
                                }
                                __syncwarp();
                            }
                        }
                    }
                };
                // 32 columns are on their way while the 32 before them are worked on
                uint32_t v0[32], v1[32];
                if (w.kblocks) {
                    tmem_load(acc, v0);
                } else {
#pragma unroll
                    for (int j = 0; j < 32; j++) v0[j] = v1[j] = 0;
                }
#pragma unroll 1
                for (int c = 0; c < 4; c += 2) {
                    if (w.kblocks) {
                        tmem_wait(v0);
                        tmem_load(acc + 32 * (c + 1), v1);
                    }
                    take(c, v0);
                    if (w.kblocks) {
                        tmem_wait(v1);
                        if (c == 0) tmem_load(acc + 64, v0);
                        else release();
                    }
                    take(c + 1, v1);
                }
            }
            if (w.kblocks) tile++;
        }
        if (KIND != kStats && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    pair_sync<CG>();                             // neither block of a pair leaves while the other may still signal it
    if (warp == 2) {
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// ------------------------------------------------------------------------------------------------ joins

__global__ void __launch_bounds__(256) rd_vocab_join_kernel(JoinParams p)
{
    pdl_start();
    const uint32_t in_band = blockIdx.x * 8 + (threadIdx.x >> 5), row = p.row0 + in_band;
    const int lane = threadIdx.x & 31;
    if (in_band >= p.rows_most || row >= (p.rows.direct ? p.n : p.meta->m)) return;
    bool counts;
    const int label = p.rows.label_row(row, counts);
    const float2 x = join_row(p.part + size_t(in_band) * p.parts, p.parts, lane);
    write_row(x, counts, label >= 0 ? p.packed_target[row] : 0.0f, p.z, p.rows.token(row), lane, p.loss, p.lse, p.target);
}

// ------------------------------------------------------------------------------------------------ loss of a few tokens

// One token, as when a server scores what it generates, and up to four on a weight that TMA cannot address: the weight's bytes are
// all that counts, so no tensor cores, but warps that stream four rows of the weight at a time past the hidden rows in shared memory.
// B200, us, tensor cores / this: 1 token of 131072 x 4096 168.9 / 159.6, 131072 x 256 22.4 / 17.4, 32768 x 1024 19.2 / 16.7, 8192 x 4096
// 22.4 / 17.1, 4096 x 512 11.3 / 7.1, 1009 x 256 8.5 / 7.4; of 32768 x 1024 2 tokens 17.9 / 19.2, 4 17.6 / 27.6; dim 1001, which the
// tensor cores need a copy for: 1 token 74 / 32 to 37, 4 75 / 40 to 50.
constexpr size_t kFewTokens = 4;
constexpr size_t kFewBytes = 32768;       // of hidden rows in shared memory
constexpr int kFewRows = 4;
constexpr unsigned kFewBlocks = 148 * 3;  // what fits at once

struct FewParams {
    const uint16_t *hidden, *weight;
    const void *labels;
    size_t hidden_stride, weight_stride;
    uint32_t n, rows, dim;
    long long first;
    bool wide_labels;
    float scale, scale2, z;
    float2 *part;             // [token][thread block]
    float *packed_target;     // per token
    uint32_t parts;
    float *loss, *lse, *target;
};

template <bool BF16> __device__ __forceinline__ float2 widen2(uint32_t v)
{
    if (BF16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}

// V: elements per access, 8 or 1.  N: tokens, with room to spare.
template <bool BF16, int V, int N> __global__ void __launch_bounds__(256, 3) rd_vocab_few_kernel(FewParams p)
{
    extern __shared__ __align__(16) unsigned char few_smem[];
    uint16_t *h = reinterpret_cast<uint16_t *>(few_smem);            // N rows of `padded` elements, zeros behind dim
    __shared__ float2 warp_part[8][N];
    pdl_wait_first();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t padded = (p.dim + 7) / 8 * 8;
    int label[N];
#pragma unroll
    for (int t = 0; t < N; t++) {
        const long long l = t < int(p.n) ? label_of(p.labels, p.wide_labels, t) : -1;
        label[t] = l >= p.first && l - p.first < static_cast<long long>(p.rows) ? int(l - p.first) : -1;
        for (uint32_t j = threadIdx.x; j < padded; j += 256) h[t * padded + j] = t < int(p.n) && j < p.dim ? p.hidden[t * p.hidden_stride + j] : uint16_t(0);
    }
    __syncthreads();
    float top[N], sum[N];
#pragma unroll
    for (int t = 0; t < N; t++) top[t] = -INFINITY, sum[t] = 0.0f;
    // an equal share of the rows for every warp; in its last turn the rows it lacks are its last one again, which costs no memory traffic
    const uint32_t warps = gridDim.x * 8, self = blockIdx.x * 8 + warp, end = uint32_t(uint64_t(p.rows) * (self + 1) / warps);
    for (uint32_t r0 = uint32_t(uint64_t(p.rows) * self / warps); r0 < end; r0 += kFewRows) {
        const uint16_t *row[kFewRows];
#pragma unroll
        for (int r = 0; r < kFewRows; r++) row[r] = p.weight + size_t(min(r0 + r, end - 1)) * p.weight_stride;
        float acc[kFewRows][N] = {};
        if (V == 8) {
#pragma unroll 2
            for (uint32_t j = lane * 8; j < p.dim; j += 256) {
                uint4 x[kFewRows];
#pragma unroll
                for (int r = 0; r < kFewRows; r++) x[r] = __ldg(reinterpret_cast<const uint4 *>(row[r] + j));
#pragma unroll
                for (int t = 0; t < N; t++) {
                    const uint4 y = *reinterpret_cast<const uint4 *>(h + t * padded + j);
                    const float2 y0 = widen2<BF16>(y.x), y1 = widen2<BF16>(y.y), y2 = widen2<BF16>(y.z), y3 = widen2<BF16>(y.w);
#pragma unroll
                    for (int r = 0; r < kFewRows; r++) {
                        const float2 x0 = widen2<BF16>(x[r].x), x1 = widen2<BF16>(x[r].y), x2 = widen2<BF16>(x[r].z), x3 = widen2<BF16>(x[r].w);
                        float a = acc[r][t];
                        a = fmaf(x0.x, y0.x, a), a = fmaf(x0.y, y0.y, a), a = fmaf(x1.x, y1.x, a), a = fmaf(x1.y, y1.y, a);
                        a = fmaf(x2.x, y2.x, a), a = fmaf(x2.y, y2.y, a), a = fmaf(x3.x, y3.x, a), a = fmaf(x3.y, y3.y, a);
                        acc[r][t] = a;
                    }
                }
            }
        } else {
#pragma unroll 4
            for (uint32_t j = lane; j < p.dim; j += 32) {
#pragma unroll
                for (int r = 0; r < kFewRows; r++) {
                    const float x = widen2<BF16>(row[r][j]).x;
#pragma unroll
                    for (int t = 0; t < N; t++) acc[r][t] = fmaf(x, widen2<BF16>(h[t * padded + j]).x, acc[r][t]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < N; t++) {
            float most = top[t], y[kFewRows];
#pragma unroll
            for (int r = 0; r < kFewRows; r++) {
                float a = acc[r][t];
#pragma unroll
                for (int d = 16; d; d /= 2) a += __shfl_xor_sync(0xffffffffu, a, d);
                if (r0 + r < end && r0 + r == uint32_t(label[t]) && lane == 0) p.packed_target[t] = a * p.scale;
                y[r] = r0 + r < end ? a * p.scale2 : -INFINITY;
                most = fmaxf(most, y[r]);
            }
            // an infinite maximum must not meet itself in a difference
            const float ref = fabsf(most) == INFINITY ? 0.0f : most;
            float s = fabsf(top[t]) == INFINITY ? sum[t] : sum[t] * exp2_fast(top[t] - ref);
#pragma unroll
            for (int r = 0; r < kFewRows; r++) s += exp2_fast(y[r] - ref);
            sum[t] = s;
            top[t] = most;
        }
    }
    if (lane == 0) {
#pragma unroll
        for (int t = 0; t < N; t++) warp_part[warp][t] = make_float2(top[t], sum[t]);
    }
    __syncthreads();
    if (warp == 0 && lane < 8) {
#pragma unroll
        for (int t = 0; t < N; t++) {
            float2 x = warp_part[lane][t];
#pragma unroll
            for (int d = 4; d; d /= 2) join_parts(x, make_float2(__shfl_down_sync(0xffu, x.x, d), __shfl_down_sync(0xffu, x.y, d)));
            if (lane == 0 && t < int(p.n)) p.part[size_t(t) * p.parts + blockIdx.x] = x;
        }
    }
}

// A thread block per token.
__global__ void __launch_bounds__(128) rd_vocab_few_join_kernel(FewParams p)
{
    __shared__ float2 of_warp[4];
    // the labels are the caller's: the kernel before this one has seen them there before it let this one start
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t t = blockIdx.x;
    const long long l = label_of(p.labels, p.wide_labels, t);
    const bool here = l >= p.first && l - p.first < static_cast<long long>(p.rows);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float target = here ? p.packed_target[t] : 0.0f;
    float2 x = make_float2(-INFINITY, 0.0f), y[(kFewBlocks + 127) / 128];
#pragma unroll
    for (uint32_t k = 0; k < sizeof(y) / sizeof(y[0]); k++)
        y[k] = threadIdx.x + 128 * k < p.parts ? p.part[size_t(t) * p.parts + threadIdx.x + 128 * k] : make_float2(-INFINITY, 0.0f);
#pragma unroll
    for (uint32_t k = 0; k < sizeof(y) / sizeof(y[0]); k++) join_parts(x, y[k]);
#pragma unroll
    for (int d = 16; d; d /= 2) join_parts(x, make_float2(__shfl_down_sync(0xffffffffu, x.x, d), __shfl_down_sync(0xffffffffu, x.y, d)));
    if (lane == 0) of_warp[warp] = x;
    __syncthreads();
    if (warp) return;
#pragma unroll
    for (int k = 1; k < 4; k++) join_parts(x, of_warp[k]);
    write_row(x, l >= 0, target, p.z, t, lane, p.loss, p.lse, p.target);
}

struct FinishParams {
    const float *dh;
    Rows rows;
    const Meta *meta;
    size_t dh_rows, dh_stride, out_stride;
    uint32_t dim, splits;
    uint16_t *out;
    bool wide;
};

constexpr uint32_t kFinishColumns = 1024;         // per thread block: 256 threads with four each

// Adds the parts of dh in order, takes the power of two off and rounds.
template <bool BF16> __global__ void __launch_bounds__(256) rd_vocab_finish_kernel(FinishParams p)
{
    pdl_start();
    const uint32_t j = blockIdx.y * kFinishColumns + threadIdx.x * 4;
    const uint32_t m = p.meta->m;
    const float unboost = p.meta->unboost;
    if (j >= p.dim) return;
    const size_t step = p.dh_rows * p.dh_stride;
    for (uint32_t row = blockIdx.x; row < m; row += gridDim.x) {
        const float *src = p.dh + size_t(row) * p.dh_stride + j;        // rows hold a multiple of 8 values
        uint16_t *dst = p.out + p.rows.token(row) * p.out_stride + j;
        const bool counts = p.rows.counts(row);            // else zeros, whatever the weight holds
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (uint32_t s = 0; s < p.splits; s++) {
            const float4 x = *reinterpret_cast<const float4 *>(src + s * step);
            sum.x += x.x;
            sum.y += x.y;
            sum.z += x.z;
            sum.w += x.w;
        }
        const uint32_t lo = counts ? pack2<BF16>(sum.x * unboost, sum.y * unboost) : 0, hi = counts ? pack2<BF16>(sum.z * unboost, sum.w * unboost) : 0;
        if (p.wide && j + 4 <= p.dim) {
            *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
        } else {
            const uint16_t v[4] = {uint16_t(lo), uint16_t(lo >> 16), uint16_t(hi), uint16_t(hi >> 16)};
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (j + k < p.dim) dst[k] = v[k];
        }
    }
}

// ------------------------------------------------------------------------------------------------ host

// TMA wants 16-byte aligned rows.
bool needs_align(const VocabArgs &a) { return reinterpret_cast<uintptr_t>(a.weight) % 16 != 0 || a.weight_stride * 2 % 16 != 0; }

// Whether pairs of thread blocks compute tiles of 256 x 256: as soon as there is more than one tile of 128 tokens.  Up to there half
// of a pair's tile would be empty (both measured when pairs were brought in, with the loops of that time: gradient of 128 tokens x
// 131072 x 4096 705 us by single blocks, 866 by pairs; of 8192 tokens 22.2 ms by single blocks, 21.6 by pairs, B200).
int pair_or_single(size_t n) { return n > kRowsM ? 2 : 1; }

constexpr size_t kSms = 148;
// Tokens whose softmax statistics are kept at a time, 16 bytes for 256 logits of each: 134 MB for 131072 logits however many tokens.
constexpr size_t kBandRows = 16384;
constexpr double kFinishSteps = 9;        // what the kernel that adds up dh costs, in steps of the summed index

// Parts that the sum over a piece is cut into for dh.  More parts fill the groups of thread blocks more evenly, but each is a
// matrix of its own that is written and read once more; times in steps of the summed index (0.28 us on an SM).
size_t dh_splits(const VocabArgs &a, size_t piece)
{
    const size_t cg = pair_or_single(a.n), tile_m = kRowsM * cg, groups = kSms / cg;
    const size_t dh_n = (a.dim + kTileN - 1) / kTileN, tiles = (a.n + tile_m - 1) / tile_m * dh_n;
    const double step_bytes = 0.28e-6 * 6.5e12, k_piece = double(piece / kTileK), k_tokens = double((a.n + kTileK - 1) / kTileK);
    const double dw = double((piece + tile_m - 1) / tile_m * dh_n) * (k_tokens + kTileOverhead);
    size_t best = 1;
    double best_time = 0;
    for (size_t s = 1; s <= 64 && s * 8 <= size_t(k_piece) + 7; s++) {
        const size_t units = tiles * s;
        const double unit = double((size_t(k_piece) + s - 1) / s + kTileOverhead), even = (double(units) * unit + dw) / double(groups);
        const double longest = double((units + groups - 1) / groups) * unit;
        const bool whole = s == 1 && a.rows <= piece;          // written as it is, by no further kernel
        const double time = (even > longest ? even : longest) + (whole ? 0 : double(s) * double(a.n * a.dim) * 8 / step_bytes + kFinishSteps);
        if (s == 1 || time < best_time) best = s, best_time = time;
    }
    return best;
}

struct Layout {
    Meta *meta;
    TileCount *tiles;
    int *index, *label;
    float *gp, *gt, *lse2, *target, *dh;
    float2 *part;
    uint16_t *packed, *dx, *weight;
    size_t rows_padded, packed_stride, dx_stride, piece, splits, dh_stride, band, bytes;
};

constexpr size_t kDxBytes = size_t(256) << 20;    // what the gradient keeps of dx at a time

Layout lay_out(const VocabArgs &a, bool gradient, bool want_hidden)
{
    Layout l{};
    if (a.n == 0) return l;
    Part w(a.workspace);
    l.rows_padded = round_up(a.n, kRowPad);
    l.packed_stride = round_up(a.dim, 64);
    l.meta = w.take<Meta>(1);
    l.tiles = w.take<TileCount>((a.n + kCountTile - 1) / kCountTile);
    l.index = w.take<int>(l.rows_padded);
    l.label = w.take<int>(l.rows_padded);
    l.packed = w.take<uint16_t>(l.rows_padded * l.packed_stride);
    if (needs_align(a)) l.weight = w.take<uint16_t>(a.rows * l.packed_stride);
    if (!gradient) {
        l.target = w.take<float>(l.rows_padded);
        const size_t halves = 2 * ((a.rows + kTileN - 1) / kTileN);
        l.band = l.rows_padded < kBandRows ? l.rows_padded : kBandRows;
        l.part = w.take<float2>(l.band * (halves > kSms ? halves : kSms));           // smaller tiles: at most one per SM
    } else {
        l.gp = w.take<float>(l.rows_padded);
        l.gt = w.take<float>(l.rows_padded);
        l.lse2 = w.take<float>(l.rows_padded);
        const size_t most = kDxBytes / (l.rows_padded * 2) / kTileN * kTileN;
        l.piece = round_up(a.rows, kTileN);
        if (l.piece > most) l.piece = most < 1024 ? 1024 : most;
        if (l.piece > round_up(a.rows, kTileN)) l.piece = round_up(a.rows, kTileN);
        l.dx_stride = l.piece;
        l.dx = w.take<uint16_t>(l.rows_padded * l.dx_stride);
        l.dh_stride = l.packed_stride;
        l.splits = want_hidden ? dh_splits(a, l.piece) : 1;
        if (want_hidden && (l.splits > 1 || a.rows > l.piece)) l.dh = w.take<float>(l.splits * a.n * l.dh_stride);
    }
    l.bytes = w.at;
    return l;
}

template <int KIND, bool BF16, int CG> cudaError_t launch_mma(const MmaParams &p, int device, size_t most_units, cudaStream_t stream)
{
    constexpr uint32_t smem = Shape<KIND, CG>::smem;
    static std::atomic<bool> ready[64];
    if (device >= 64 || !ready[device].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(rd_vocab_mma_kernel<KIND, BF16, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (device < 64) ready[device].store(true, std::memory_order_release);
    }
    const size_t groups = size_t(sm_count_of(device)) / CG;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(unsigned((most_units < groups ? most_units : groups) * CG));
    c.blockDim = dim3(kMmaThreads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    cudaLaunchAttribute attrs[2] = {pdl_attribute()};
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = CG;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    c.attrs = attrs;
    c.numAttrs = 2;
    return cudaLaunchKernelEx(&c, rd_vocab_mma_kernel<KIND, BF16, CG>, p);
}
template <int KIND> cudaError_t launch_mma(const MmaParams &p, bool bf16, int cg, int device, size_t most_units, cudaStream_t stream)
{
    if (cg == 2) return bf16 ? launch_mma<KIND, true, 2>(p, device, most_units, stream) : launch_mma<KIND, false, 2>(p, device, most_units, stream);
    return bf16 ? launch_mma<KIND, true, 1>(p, device, most_units, stream) : launch_mma<KIND, false, 1>(p, device, most_units, stream);
}

// Whether the products read the hidden rows where they lie: one tile of tokens, in rows that TMA can address.
bool is_direct(const VocabArgs &a) { return a.n <= kRowsM && reinterpret_cast<uintptr_t>(a.hidden) % 16 == 0 && a.hidden_stride % 8 == 0 && a.hidden_stride > 0; }

// Counting and packing, and the weight's aligned copy where one is needed.
cudaError_t prepare(const VocabArgs &a, const Layout &l, bool gradient, const uint16_t **weight, size_t *weight_stride)
{
    cudaError_t e = cudaSuccess;
    *weight = static_cast<const uint16_t *>(a.weight);
    *weight_stride = a.weight_stride;
    if (l.weight) {
        e = launch(rd_vocab_align_kernel, 1184, kPackThreads, a.stream, l.weight, uint32_t(l.packed_stride), *weight, a.weight_stride, a.rows, uint32_t(a.dim));
        *weight = l.weight;
        *weight_stride = l.packed_stride;
    }
    if (e != cudaSuccess || is_direct(a)) return e;
    PackParams p{};
    p.hidden = static_cast<const uint16_t *>(a.hidden);
    p.labels = a.labels;
    p.hidden_stride = a.hidden_stride;
    p.n = a.n;
    p.rows = a.rows;
    p.dim = uint32_t(a.dim);
    p.packed_stride = uint32_t(l.packed_stride);
    p.first = a.first_row;
    p.wide_labels = a.wide_labels;
    p.copy16 = reinterpret_cast<uintptr_t>(a.hidden) % 16 == 0 && a.hidden_stride % 8 == 0 && a.dim % 8 == 0;
    p.scale = a.scale;
    p.z = a.z_loss;
    p.packed = l.packed;
    p.index = l.index;
    p.label = l.label;
    p.tiles = l.tiles;
    p.meta = l.meta;
    p.loss = a.loss;
    p.lse_out = a.lse_out;
    p.target = a.target;
    p.lse = a.lse;
    p.grad_loss = a.grad_loss;
    p.grad_loss_stride = a.grad_loss_stride;
    p.gp = l.gp;
    p.gt = l.gt;
    p.lse2 = l.lse2;
    p.grad_hidden = static_cast<uint16_t *>(a.grad_hidden);
    p.grad_hidden_stride = a.grad_hidden_stride;
    p.gradient = gradient;
    p.fp16 = !a.bf16;
    unsigned tiles = 0;
    if (a.n >= kCountFrom) {
        tiles = unsigned((a.n + kCountTile - 1) / kCountTile);
        e = launch(rd_vocab_count_kernel, tiles, kCountTile, a.stream, p, l.tiles);
        if (e != cudaSuccess) return e;
    }
    // few tokens: a thread block for each, so that their rows are copied by many threads
    if (a.n <= 1024) {
        const unsigned blocks = unsigned(a.n);
        e = launch(rd_vocab_pack_kernel<1>, blocks + (gradient ? kZeroPad : 0), kPackThreads, a.stream, p, blocks, tiles);
    } else {
        const unsigned blocks = unsigned((a.n + 7) / 8);
        e = launch(rd_vocab_pack_kernel<8>, blocks + (gradient ? kZeroPad / 8 : 0), kPackThreads, a.stream, p, blocks, tiles);
    }
    return e;
}

// Token tiles that go over the vocabulary together: their hidden rows (tile x dim) should stay in L2 beside the weight's.
uint32_t token_group(size_t dim, size_t tile_m)
{
    const size_t g = (size_t(32) << 20) / (tile_m * dim * 2);
    return uint32_t(g < 1 ? 1 : g > 64 ? 64 : g);
}

// Rows of a left operand that a thread block brings in: all 128, or as many as there are tokens.
size_t a_rows(size_t n) { return n < kRowsM ? round_up(n, 8) : kRowsM; }

Rows rows_of(const VocabArgs &a, const Layout &l) { return Rows{l.index, l.label, a.labels, a.first_row, a.rows, is_direct(a), a.wide_labels}; }

// The hidden rows as the logits' left operand.
bool encode_hidden(CUtensorMap *map, const VocabArgs &a, const Layout &l)
{
    return is_direct(a) ? encode(map, a.bf16, a.hidden, a.dim, a.n, a.hidden_stride, uint32_t(a_rows(a.n)))
                        : encode(map, a.bf16, l.packed, a.dim, l.rows_padded, l.packed_stride, uint32_t(a_rows(a.n)));
}

// Columns of the logits' tiles: 256, or fewer where that leaves half of the thread blocks (pairs) without a tile.
uint32_t tile_columns(size_t tiles_m, size_t rows, int cg)
{
    size_t n = kTileN;
    while (n > 64 && tiles_m * ((rows + n - 1) / n) * 2 <= kSms / cg) n /= 2;
    return uint32_t(n);
}

template <int KIND> void set_ring(MmaParams &q, int cg)
{
    const Ring r = ring_of(cg == 2 ? Shape<KIND, 2>::ring : Shape<KIND, 1>::ring, q.a_rows, q.tile_n / uint32_t(cg));
    q.stage = r.stage;
    q.stages = r.stages;
}

void common(MmaParams &q, const VocabArgs &a, const Layout &l, int cg)
{
    q.meta = l.meta;
    q.rows = rows_of(a, l);
    q.direct.n = uint32_t(a.n);
    q.dim = uint32_t(a.dim);
    q.group = token_group(a.dim, size_t(kRowsM) * cg);
    q.a_rows = uint32_t(a_rows(a.n));
    q.scale = a.scale;
    q.scale2 = a.scale * kLog2e;
}

bool is_few(const VocabArgs &a) { return a.n <= (needs_align(a) ? kFewTokens : 1) && a.n * round_up(a.dim, 8) * 2 <= kFewBytes; }

template <bool BF16, int V, int N> cudaError_t launch_few(const VocabArgs &a, const FewParams &p, unsigned blocks)
{
    cudaLaunchConfig_t c{};
    cudaLaunchAttribute pdl = pdl_attribute();
    c.gridDim = dim3(blocks);
    c.blockDim = dim3(256);
    c.dynamicSmemBytes = unsigned(N * round_up(a.dim, 8) * 2);
    c.stream = a.stream;
    c.attrs = &pdl;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, rd_vocab_few_kernel<BF16, V, N>, p);
}
template <bool BF16> cudaError_t launch_few(const VocabArgs &a, const FewParams &p, unsigned blocks)
{
    // TMA's alignment and whole words of 16 bytes
    if (!needs_align(a) && a.dim % 8 == 0) return launch_few<BF16, 8, 1>(a, p, blocks);
    return a.n == 1 ? launch_few<BF16, 1, 1>(a, p, blocks) : a.n == 2 ? launch_few<BF16, 1, 2>(a, p, blocks) : launch_few<BF16, 1, 4>(a, p, blocks);
}

cudaError_t vocab_loss_few(const VocabArgs &a)
{
    Part w(a.workspace);
    const unsigned wanted = unsigned((a.rows + 8 * kFewRows - 1) / (8 * kFewRows)), blocks = wanted < kFewBlocks ? wanted : kFewBlocks;
    FewParams p{};
    p.hidden = static_cast<const uint16_t *>(a.hidden);
    p.weight = static_cast<const uint16_t *>(a.weight);
    p.labels = a.labels;
    p.hidden_stride = a.hidden_stride;
    p.weight_stride = a.weight_stride;
    p.n = uint32_t(a.n);
    p.rows = uint32_t(a.rows);
    p.dim = uint32_t(a.dim);
    p.first = a.first_row;
    p.wide_labels = a.wide_labels;
    p.scale = a.scale;
    p.scale2 = a.scale * kLog2e;
    p.z = a.z_loss;
    p.part = w.take<float2>(kFewTokens * kFewBlocks);
    p.packed_target = w.take<float>(kFewTokens);
    p.parts = blocks;
    p.loss = a.loss;
    p.lse = a.lse_out;
    p.target = a.target;
    const cudaError_t e = a.bf16 ? launch_few<true>(a, p, blocks) : launch_few<false>(a, p, blocks);
    if (e != cudaSuccess) return e;
    return launch(rd_vocab_few_join_kernel, unsigned(a.n), 128, a.stream, p);
}

}  // namespace

size_t vocab_loss_workspace(const VocabArgs &a)
{
    return is_few(a) && a.n ? 1024 * (round_up(kFewTokens * kFewBlocks * sizeof(float2), 1024) / 1024 + 1) : lay_out(a, false, false).bytes;
}

cudaError_t vocab_loss(const VocabArgs &a)
{
    if (is_few(a)) return vocab_loss_few(a);
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const int cg = pair_or_single(a.n);
    const size_t tile_m = size_t(kRowsM) * cg;
    const Layout l = lay_out(a, false, false);
    const uint16_t *weight;
    size_t weight_stride;
    e = prepare(a, l, false, &weight, &weight_stride);
    if (e != cudaSuccess) return e;
    MmaParams q{};
    common(q, a, l, cg);
    const size_t tiles_m = (a.n + tile_m - 1) / tile_m;
    q.tile_n = tile_columns(tiles_m, a.rows, cg);
    set_ring<kStats>(q, cg);
    const size_t tiles_n = (a.rows + q.tile_n - 1) / q.tile_n;
    if (!encode_hidden(&q.a_k, a, l) || !encode(&q.b_k, a.bf16, weight, a.dim, a.rows, weight_stride, q.tile_n / cg)) return cudaErrorInvalidValue;
    q.part = l.part;
    q.parts = uint32_t(q.tile_n == kTileN ? 2 * tiles_n : tiles_n);
    q.target = l.target;
    q.piece0 = 0;
    q.piece = uint32_t(a.rows);
    for (size_t row0 = 0; row0 < a.n; row0 += l.band) {
        const size_t rows = a.n - row0 < l.band ? a.n - row0 : l.band;
        q.row0 = uint32_t(row0);
        q.rows_most = uint32_t(rows);
        e = launch_mma<kStats>(q, a.bf16, cg, device, (rows + tile_m - 1) / tile_m * tiles_n, a.stream);
        if (e != cudaSuccess) return e;
        const JoinParams j{l.part, l.target, q.rows, l.meta, uint32_t(a.n), q.row0, q.rows_most, q.parts, a.z_loss,
                           a.loss, a.lse_out, a.target};
        e = launch(rd_vocab_join_kernel, unsigned((rows + 7) / 8), 256, a.stream, j);
        if (e != cudaSuccess) return e;
    }
    return e;
}

size_t vocab_loss_grad_workspace(const VocabArgs &a, bool want_hidden) { return lay_out(a, true, want_hidden).bytes; }

cudaError_t vocab_loss_grad(const VocabArgs &a)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const int cg = pair_or_single(a.n);
    const size_t tile_m = size_t(kRowsM) * cg;
    const Layout l = lay_out(a, true, a.grad_hidden != nullptr);
    const uint16_t *weight;
    size_t weight_stride;
    e = prepare(a, l, true, &weight, &weight_stride);
    if (e != cudaSuccess) return e;
    MmaParams logits{}, grads{};
    common(logits, a, l, cg);
    common(grads, a, l, cg);
    logits.gp = l.gp;
    logits.gt = l.gt;
    logits.lse2 = l.lse2;
    grads.dh_stride = l.dh_stride;
    grads.splits = uint32_t(l.splits);
    grads.dw = static_cast<uint16_t *>(a.grad_weight);
    grads.dw_stride = a.grad_weight_stride;
    grads.dw_tma = reinterpret_cast<uintptr_t>(a.grad_weight) % 16 == 0 && a.grad_weight_stride % 8 == 0;
    grads.want_dh = a.grad_hidden != nullptr;
    grads.want_dw = a.grad_weight != nullptr;
    const size_t tiles_m = (a.n + tile_m - 1) / tile_m, tiles_d = (a.dim + kTileN - 1) / kTileN;
    logits.tile_n = tile_columns(tiles_m, a.rows < l.piece ? a.rows : l.piece, cg);
    set_ring<kDlogits>(logits, cg);
    if (is_direct(a))
        logits.direct = Direct{uint32_t(a.n), static_cast<const uint16_t *>(a.hidden), a.hidden_stride, a.grad_weight ? l.packed : nullptr, uint32_t(l.packed_stride), a.lse,
                               a.grad_loss, a.grad_loss_stride, a.scale, a.z_loss, l.meta, a.dim % 8 == 0};
    if (!encode_hidden(&logits.a_k, a, l) || !encode(&logits.b_k, a.bf16, weight, a.dim, a.rows, weight_stride, logits.tile_n / cg) ||
        !encode(&grads.a_k, a.bf16, l.dx, l.dx_stride, l.rows_padded, l.dx_stride, uint32_t(a_rows(a.n))) || !encode(&grads.a_mn, a.bf16, l.dx, l.dx_stride, l.rows_padded, l.dx_stride, 64) ||
        !encode(&logits.dx_out, a.bf16, l.dx, l.dx_stride, l.rows_padded, l.dx_stride, 32) || !encode(&grads.b_mn, a.bf16, weight, a.dim, a.rows, weight_stride, 64) || !encode(&grads.b2_mn, a.bf16, l.packed, a.dim, l.rows_padded, l.packed_stride, 64))
        return cudaErrorInvalidValue;
    const bool whole = l.splits == 1 && a.rows <= l.piece;
    if (grads.want_dh && whole) {
        grads.gh = static_cast<uint16_t *>(a.grad_hidden);
        grads.gh_stride = a.grad_hidden_stride;
        grads.gh_wide = reinterpret_cast<uintptr_t>(a.grad_hidden) % 16 == 0 && a.grad_hidden_stride % 8 == 0;
    }
    if (grads.want_dh && !whole && !encode_dh(&grads.dh_out, l.dh, l.dh_stride, a.n, l.splits)) return cudaErrorInvalidValue;
    if (grads.want_dw && grads.dw_tma && !encode(&grads.dw_out, a.bf16, a.grad_weight, a.dim, a.rows, a.grad_weight_stride, 32)) return cudaErrorInvalidValue;
    for (size_t v = 0; v < a.rows; v += l.piece) {
        const size_t piece = a.rows - v < l.piece ? a.rows - v : l.piece;
        logits.piece0 = grads.piece0 = uint32_t(v);
        logits.piece = grads.piece = uint32_t(piece);
        logits.first_piece = grads.first_piece = v == 0;
        e = launch_mma<kDlogits>(logits, a.bf16, cg, device, tiles_m * ((piece + logits.tile_n - 1) / logits.tile_n), a.stream);
        if (e != cudaSuccess) return e;
        const size_t units = (grads.want_dh ? tiles_m * tiles_d * l.splits : 0) + (grads.want_dw ? (piece + tile_m - 1) / tile_m * tiles_d : 0);
        e = launch_mma<kGrads>(grads, a.bf16, cg, device, units, a.stream);
        if (e != cudaSuccess) return e;
    }
    if (a.grad_hidden && !whole) {
        const bool wide = reinterpret_cast<uintptr_t>(a.grad_hidden) % 8 == 0 && a.grad_hidden_stride % 4 == 0;
        const FinishParams f{l.dh, grads.rows, l.meta, a.n, l.dh_stride, a.grad_hidden_stride, uint32_t(a.dim), uint32_t(l.splits), static_cast<uint16_t *>(a.grad_hidden), wide};
        const dim3 grid(unsigned(a.n < 65536 ? a.n : 65536), unsigned((a.dim + kFinishColumns - 1) / kFinishColumns));
        e = a.bf16 ? launch(rd_vocab_finish_kernel<true>, grid, 256, a.stream, f) : launch(rd_vocab_finish_kernel<false>, grid, 256, a.stream, f);
    }
    return e;
}

cudaError_t vocab_status(int *status)
{
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return e;
    int of_embed = 0;
    e = embed_status(&of_embed);
    if (e != cudaSuccess) return e;
    e = cudaMemcpyFromSymbol(status, g_wait_status, sizeof(int));
    if (e != cudaSuccess) return e;
    const int zero = 0;
    if (*status) e = cudaMemcpyToSymbol(g_wait_status, &zero, sizeof(int));
    *status |= of_embed;
    return e;
}

}  // namespace rd
