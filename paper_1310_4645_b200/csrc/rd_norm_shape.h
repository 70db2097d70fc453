// What the norm's host code and its kernels share: parameters, how rows are dealt out, launches by the rows' type.
#ifndef RD_NORM_SHAPE_H_
#define RD_NORM_SHAPE_H_

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace rd {

constexpr int kThreads = 256, kWarps = kThreads / 32;       // of a block: whose warps have rows of their own, or at most
constexpr uint32_t kBlockUnits = 1024;    // units of 8 columns of a row that a thread block has at most
constexpr int kUnits = 4;                 // units that a thread has at most
constexpr size_t kDropoutBlocks = 6;      // of dropout alone, an SM
constexpr int kShortBlocks = 4;           // of short rows, an SM
constexpr uint32_t kSumColumns = 16;      // of grad_weight, that a block sums up where rows are few
constexpr uint32_t kMostStages = 8;
constexpr size_t kRingBytes = 200 << 10;  // of an SM's shared memory that rows on their way may take
constexpr size_t kSms = 148;

// Types of values.
struct F32 {
    static constexpr int words = 8;       // of 8 values
};
struct B16 {
    static constexpr int words = 4;
};
struct H16 {
    static constexpr int words = 4;
};

// Dropout, as the kernels want it.
constexpr int kRounds = 10;
struct DropKeys {
    uint32_t border, border16;                // border16: border << 16
    float keep;
    uint32_t key[2 * kRounds];                // both key words of every round
    uint32_t offset0, offset1, first;
};

// The ring of stages that rows come in through.
struct RowRing {
    uint32_t stages, stage;   // how many, and bytes of one
};

struct NormParams {
    RowRing ring;
    const void *x, *residual, *weight;
    void *out, *sum;
    float *out_scale, *rstd;
    size_t x_stride, residual_stride, out_stride, sum_stride, n;
    uint32_t dim, units, per_block, blocks, threads;
    float eps, inv_dim;
    DropKeys drop;
    bool out8, release_early;
};

struct NormGradParams {
    RowRing ring;
    const void *grad_out, *sum, *weight, *grad_sum;
    const float *rstd;
    void *grad_x, *grad_residual;
    float *part;              // [groups][dim]: every group's part of grad_weight; null where it is not wanted, or summed up by columns
    void *grad_weight;        // by columns: blocks beyond row_blocks
    uint32_t row_blocks;
    size_t grad_out_stride, sum_stride, grad_sum_stride, grad_x_stride, grad_residual_stride, n;
    uint32_t dim, units, per_block, blocks, threads;
    float inv_dim;
    DropKeys drop;
    bool want_rows, release_early;
};

// How a row is dealt out, brought in and how many rows at a time.
//   Rows of up to 32 units have 8, 16 or 32 lanes of a warp each and no ring: those would be copies of a few hundred bytes (262144 x 128
//   bf16 by a warp a row and a ring 81 us, gradient 145; so 44 and 50).
//   A warp has a row if it holds it with four units a thread, two without a ring; else as few warps of a thread block as hold it, or a
//   cluster of up to eight blocks, as few as do: their meetings cost more than blocks an SM gain (gradient of 8192 x 16384 bf16 by two
//   blocks 245 us, by four 430).
//   Four units a thread: then the join of a row costs few instructions a value.  Two, and twice the warps, in the gradient (few) while one
//   block of them holds a block's part (16384 x 4096 bf16 with dropout 129 us, with four 137), and without a ring, where operands
//   stay in registers (16384 x 4095 bf16 norm 195 us, with four 233; gradient 210 and 269), but for norms of more than 8192 columns
//   (4096 x 10001: 168 us, in four blocks with two units 228, with four and 80 registers 211).
//   As many groups (a block of warps with a row each, or the blocks of one row) as registers (80 a thread, 128 with four units and no ring)
//   and shared memory with two stages or more allow.  (All B200.)
// unit_bytes: of all matrices that come in by the ring, for 8 columns; 0: none does.
struct RowDeal {
    uint32_t units, per_block, blocks, threads;
    int nv;                   // units a thread
    int lanes;                // short rows: the lanes that have one; 0: others
    bool warp;
    bool full() const { return size_t(blocks) * per_block == units && per_block == (warp ? 32 : threads) * uint32_t(nv); }
};
inline RowDeal deal(size_t dim, size_t unit_bytes, bool few)
{
    RowDeal d{};
    d.units = uint32_t((dim + 7) / 8);
    d.blocks = 1;
    d.threads = kThreads;
    d.per_block = d.units;
    const int most = unit_bytes ? kUnits : kUnits / 2;
    if (unit_bytes && d.units <= 32) {
        d.warp = true;
        d.nv = 1;
        d.lanes = d.units <= 8 ? 8 : d.units <= 16 ? 16 : 32;
        return d;
    }
    if (d.units <= uint32_t(32 * most)) {
        d.warp = true;
        d.nv = most;
        while (d.nv > 2 && d.units <= uint32_t(16 * d.nv)) d.nv /= 2;
        return d;
    }
    auto part = [&] { return (d.units + d.blocks - 1) / d.blocks; };
    while (d.blocks < 8 && part() > (unit_bytes || (!few && d.units > kBlockUnits) ? kBlockUnits : kBlockUnits / 2)) d.blocks *= 2;
    // whole warps' columns, so that no 256 columns are two blocks'; then perhaps fewer blocks, none without columns
    d.per_block = (part() + 31) / 32 * 32;
    d.blocks = (d.units + d.per_block - 1) / d.per_block;
    d.nv = (few || !unit_bytes) && d.per_block <= uint32_t(kThreads * kUnits / 2) ? kUnits / 2 : kUnits;
    d.threads = (d.per_block + 32 * d.nv - 1) / (32 * d.nv) * 32;
    return d;
}

struct RowShape {
    size_t groups, smem;
    bool one_turn;            // no group has more than one row
    RowRing ring;
};
inline RowShape shape_of(size_t n, const RowDeal &d, size_t unit_bytes)
{
    RowShape s{};
    const size_t rows = d.lanes ? kWarps * 32 / d.lanes : d.warp ? kWarps : 1, wanted = (n + rows - 1) / rows;
    size_t per_sm = 65536 / (d.threads * (unit_bytes || d.nv < kUnits ? 80 : 128));
    if (d.lanes) {
        per_sm = kShortBlocks;
    } else if (unit_bytes) {
        const size_t stage = d.per_block * unit_bytes, all = stage * rows;
        while (per_sm > 1 && kRingBytes / per_sm / all < 2) per_sm--;
        const size_t fit = kRingBytes / per_sm / all;
        s.ring = RowRing{uint32_t(fit < kMostStages ? fit : kMostStages), uint32_t(stage)};
        s.smem = s.ring.stages * all;
    }
    const size_t most = kSms * per_sm / d.blocks;
    s.groups = wanted < most ? wanted : most;
    s.one_turn = wanted <= most;
    return s;
}

// A launch, besides the kernel's parameters.
struct NormCall {
    bool spread;
    RowDeal deal;
    RowShape shape;
    int sum_dtype, weight_dtype;
    cudaStream_t stream;
    size_t more_blocks;       // behind those that have rows
};
template <class T> cudaError_t launch_norm(const NormParams &p, const NormCall &c);
template <class T> cudaError_t launch_norm_grad(const NormGradParams &p, const NormCall &c);
// The word in which a file's kernels note a wait that they gave up, cleared.
template <class T> cudaError_t norm_rows_status(int *status);

}  // namespace rd

#endif  // RD_NORM_SHAPE_H_
