// sm_100a kernels of the root-mean-square norm with the residual's addition and dropout, of its gradient, and of dropout alone.
//
//   s = residual + keep x,   r = 1 / sqrt(mean s^2 + eps),   out = s r w          (8 bits: scale = max |out| / 448, out / scale)
//   xhat = s r,  g = grad_out w:   grad = r (g - xhat mean(g xhat)) + grad_sum,   grad_x = keep grad,   grad_w = sum over rows of grad_out xhat
//
// keep is 65536 / (65536 - border) where a value's 16 random bits reach the border, else 0.  The bits are those of Philox 4x32 with
// 10 rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), whose counter is the value's place:
// (column / 8, row, offset), key: the seed.  So a mask is never stored; whoever knows the place knows the bits.
//
// A row is held by 8, 16 or 32 lanes (up to 256 values), a warp (up to 1024), a thread block (up to 8192) or a cluster of up to eight of them, whose partial sums meet in
// each other's shared memory.  Everything is read and written once, the weight and, in the gradient, a row in shared memory excepted.
// What bounds it (B200): the memory, at 0.80 to 0.92 of the rate of a copy: 16384 x 4096 bf16 with dropout and residual 89 to 102 us for 537 MB,
// gradient 114 to 125 for 671, dropout alone 45 to 50 for 268; without dropout in fp32 170 for 1074, gradient 172; 2000 x 5120 into 8 bits 18.0 to
// 20.5 for 113.  A row alone: 2.4 us, the latency of a launch, a load, a reduction and a store.
#include "rd_norm_rows.h"

namespace rd {

namespace {

// Adds up the groups' parts: 32 columns a block, each by 32 threads that take every 32nd part, then those in order.
constexpr int kJoinThreads = 1024;
template <class W> __global__ void __launch_bounds__(kJoinThreads) rd_norm_weight_kernel(void *grad_weight, const float *part, uint32_t parts, uint32_t dim)
{
    __shared__ float of_lane[32][33];
    pdl_wait();
    const uint32_t column = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
    float v = 0.0f;
    if (column < dim)
#pragma unroll 8
        for (uint32_t k = lane; k < parts; k += 32) v += part[size_t(k) * dim + column];
    pdl_release();
    of_lane[threadIdx.x & 31][lane] = v;
    __syncthreads();
    // a warp per column
    v = of_lane[lane][threadIdx.x & 31];
#pragma unroll
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    const uint32_t to = blockIdx.x * 32 + lane;
    if ((threadIdx.x & 31) == 0 && to < dim) {
        if constexpr (std::is_same_v<W, F32>) static_cast<float *>(grad_weight)[to] = v;
        else if constexpr (std::is_same_v<W, B16>) static_cast<__nv_bfloat16 *>(grad_weight)[to] = __float2bfloat16_rn(v);
        else static_cast<__half *>(grad_weight)[to] = __float2half_rn(v);
    }
}

// ------------------------------------------------------------------------------------------------ dropout alone

struct DropoutParams {
    const void *x;
    void *out;
    size_t x_stride, out_stride, n;
    uint32_t dim, units, across_log;  // log2 of the threads that a row's units are dealt out to; the block's others have rows of their own
    DropKeys drop;
};

// A thread has up to two units of a row at a time.
template <class T, bool SPREAD> __global__ void __launch_bounds__(kThreads, kDropoutBlocks) rd_dropout_kernel(const __grid_constant__ DropoutParams p)
{
    using UnitT = Unit<T, SPREAD>;
    constexpr uint32_t kT = UnitT::bytes / 8;
    __shared__ uint4 bits[SPREAD ? kWarps : 1][32];
    pdl_start();
    const uint32_t across = 1u << p.across_log, x = threadIdx.x & (across - 1), y = threadIdx.x >> p.across_log, down = kThreads >> p.across_log;
    const uint32_t unit0 = blockIdx.y * across * 2 + x;
    bool has[2];
#pragma unroll
    for (int k = 0; k < 2; k++) has[k] = (SPREAD ? (unit0 + k * across) & ~31u : unit0 + k * across) < p.units;
    for (size_t row = size_t(blockIdx.x) * down + y; row < p.n; row += size_t(gridDim.x) * down) {
        const void *const from = at_byte(p.x, row * p.x_stride * kT);
        void *const to = at_byte(p.out, row * p.out_stride * kT);
        UnitT v[2];
#pragma unroll
        for (int k = 0; k < 2; k++)
            v[k].load(from, unit0 + k * across, p.dim, has[k]);
#pragma unroll
        for (int k = 0; k < 2; k++)
            if (has[k]) {
                Pair f[4];
                v[k].get(f);
                drop_values<SPREAD>(p.drop, bits[SPREAD ? threadIdx.x >> 5 : 0], unit0 + k * across, uint32_t(row), f);
                v[k].set(f);
                v[k].store(to, unit0 + k * across, p.dim);
            }
    }
}

// ------------------------------------------------------------------------------------------------ host

DropKeys drop_of(const DropArgs &d)
{
    DropKeys o{};
    o.border = d.border;
    o.border16 = d.border << 16;
    o.keep = d.keep;
    for (uint32_t i = 0; i < kRounds; i++) {
        o.key[2 * i] = uint32_t(d.seed) + i * 0x9E3779B9u;
        o.key[2 * i + 1] = uint32_t(d.seed >> 32) + i * 0xBB67AE85u;
    }
    o.offset0 = uint32_t(d.offset);
    o.offset1 = uint32_t(d.offset >> 32);
    o.first = d.first;
    return o;
}

size_t size_of(int dtype) { return dtype == RD_FP32 ? 4 : dtype == RD_E4M3 ? 1 : 2; }

// Whether a matrix's rows begin where units are one access: on multiples of 8 values' bytes, 16 at least but for 8 bits.
bool in_units(const void *p, size_t stride, int dtype)
{
    const size_t to = 8 * size_of(dtype);
    return !p || (reinterpret_cast<uintptr_t>(p) % to == 0 && stride * size_of(dtype) % to == 0);
}

// Whether grad_weight is summed up by blocks of its own beside the rows', 16 columns each, instead of from the groups' parts by another
// launch: few rows and not too many columns, which are read twice.  B200, us a call, this and the other way: 16 rows of 1000 bf16 5.1
// and 7.1, 257 of them 5.1 and 7.1, 384 6.2 and 7.4; 100 rows of 4096 5.2 and 6.9, 320 7.9 and 7.8, 384 11.0 and 8.0.
bool by_columns(size_t n, size_t dim) { return n <= 384 && n * dim <= size_t(1) << 20; }

}  // namespace

cudaError_t norm_forward(const NormArgs &a)
{
    const bool spread = a.dim % 8 != 0 || !in_units(a.x, a.x_stride, a.dtype) || !in_units(a.residual, a.residual_stride, a.sum_dtype) || !in_units(a.weight, 0, a.weight_dtype) ||
                        !in_units(a.out, a.out_stride, a.out_dtype) || !in_units(a.sum, a.sum_stride, a.sum_dtype);
    const size_t unit_bytes = spread ? 0 : 8 * (size_of(a.dtype) + (a.residual ? size_of(a.sum_dtype) : 0));
    const RowDeal d = deal(a.dim, unit_bytes, false);
    const RowShape shape = shape_of(a.n, d, unit_bytes);
    NormParams p{};
    p.ring = shape.ring;
    p.x = a.x;
    p.residual = a.residual;
    p.weight = a.weight;
    p.out = a.out;
    p.sum = a.sum;
    p.out_scale = a.out_scale;
    p.rstd = a.rstd;
    p.x_stride = a.x_stride;
    p.residual_stride = a.residual_stride;
    p.out_stride = a.out_stride;
    p.sum_stride = a.sum_stride;
    p.n = a.n;
    p.dim = uint32_t(a.dim);
    p.units = d.units;
    p.per_block = d.per_block;
    p.blocks = d.blocks;
    p.eps = a.eps;
    p.inv_dim = 1.0f / float(a.dim);
    p.drop = drop_of(a.drop);
    p.threads = d.threads;
    p.release_early = shape.one_turn;
    p.out8 = a.out_dtype == RD_E4M3;
    const NormCall call{spread, d, shape, a.sum_dtype, a.weight_dtype, a.stream, 0};
    return a.dtype == RD_FP32 ? launch_norm<F32>(p, call) : a.dtype == RD_BF16 ? launch_norm<B16>(p, call) : launch_norm<H16>(p, call);
}

size_t norm_backward_workspace(size_t n, size_t dim)
{
    if (by_columns(n, dim)) return 0;
    // a part of grad_weight of every group: the most that any types, strides and inputs give (two or three matrices of 2 or 4 bytes a value)
    size_t most = 0;
    for (const size_t unit_bytes : {0, 32, 48, 64, 80, 96}) {
        const size_t groups = shape_of(n, deal(dim, unit_bytes, true), unit_bytes).groups;
        most = groups > most ? groups : most;
    }
    return most * dim * sizeof(float);
}

cudaError_t norm_backward(const NormGradArgs &a)
{
    const bool spread = a.dim % 8 != 0 || !in_units(a.grad_out, a.grad_out_stride, a.dtype) || !in_units(a.sum, a.sum_stride, a.sum_dtype) || !in_units(a.weight, 0, a.weight_dtype) ||
                        !in_units(a.grad_sum, a.grad_sum_stride, a.sum_dtype) || !in_units(a.grad_x, a.grad_x_stride, a.dtype) ||
                        !in_units(a.grad_residual, a.grad_residual_stride, a.sum_dtype);
    const size_t unit_bytes = spread ? 0 : 8 * (size_of(a.dtype) + size_of(a.sum_dtype) * (a.grad_sum ? 2 : 1));
    RowDeal d = deal(a.dim, unit_bytes, true);
    const bool few = a.n > 0 && by_columns(a.n, a.dim), columns = few && a.grad_weight;
    // blocks that columns want; whether they are wanted or not, so that the rows' bits do not depend on it
    if (few && d.threads < kThreads) d.threads = kThreads;
    RowShape shape = shape_of(a.n, d, unit_bytes);
    // where warps have rows, their parts of grad_weight are joined in shared memory
    if (d.warp && !d.lanes && shape.smem < kWarps * a.dim * sizeof(float)) shape.smem = kWarps * a.dim * sizeof(float);
    NormGradParams p{};
    p.ring = shape.ring;
    p.grad_out = a.grad_out;
    p.sum = a.sum;
    p.weight = a.weight;
    p.grad_sum = a.grad_sum;
    p.rstd = a.rstd;
    p.grad_x = a.grad_x;
    p.grad_residual = a.grad_residual;
    p.part = a.grad_weight ? static_cast<float *>(a.workspace) : nullptr;
    p.grad_out_stride = a.grad_out_stride;
    p.sum_stride = a.sum_stride;
    p.grad_sum_stride = a.grad_sum_stride;
    p.grad_x_stride = a.grad_x_stride;
    p.grad_residual_stride = a.grad_residual_stride;
    p.n = a.n;
    p.dim = uint32_t(a.dim);
    p.units = d.units;
    p.per_block = d.per_block;
    p.blocks = d.blocks;
    p.inv_dim = 1.0f / float(a.dim);
    p.drop = drop_of(a.drop);
    p.threads = d.threads;
    p.release_early = shape.one_turn;
    p.want_rows = a.grad_x || a.grad_residual;
    p.row_blocks = uint32_t(shape.groups * d.blocks);
    if (columns) {
        p.part = nullptr;
        p.grad_weight = a.grad_weight;
    }
    auto run = [&](const NormGradParams &q, const NormCall &c) {
        return a.dtype == RD_FP32 ? launch_norm_grad<F32>(q, c) : a.dtype == RD_BF16 ? launch_norm_grad<B16>(q, c) : launch_norm_grad<H16>(q, c);
    };
    NormCall call{spread, d, shape, a.sum_dtype, a.weight_dtype, a.stream, columns ? ((a.dim + kSumColumns - 1) / kSumColumns + d.blocks - 1) / d.blocks * d.blocks : 0};
    cudaError_t e = cudaSuccess;
    bool in_place = false;        // gradients in the place of what the columns read
    for (const void *w : {a.grad_x, a.grad_residual}) in_place |= w && (w == a.grad_out || w == a.sum);
    if (columns && in_place) {
        // then the columns go first, by themselves
        NormGradParams q = p;
        NormCall c = call;
        q.row_blocks = 0;
        c.shape.groups = 0;
        e = run(q, c);
        if (e != cudaSuccess) return e;
        call.more_blocks = 0;
    }
    if (shape.groups) e = run(p, call);
    if (e != cudaSuccess || !a.grad_weight || columns) return e;
    auto *join = a.weight_dtype == RD_FP32 ? rd_norm_weight_kernel<F32> : a.weight_dtype == RD_BF16 ? rd_norm_weight_kernel<B16> : rd_norm_weight_kernel<H16>;
    return launch(join, unsigned((a.dim + 31) / 32), kJoinThreads, a.stream, a.grad_weight, static_cast<const float *>(a.workspace), uint32_t(shape.groups), uint32_t(a.dim));
}

cudaError_t norm_status(int *status)
{
    *status = 0;
    for (auto f : {norm_rows_status<F32>, norm_rows_status<B16>, norm_rows_status<H16>}) {
        int of_rows = 0;
        const cudaError_t e = f(&of_rows);
        if (e != cudaSuccess) return e;
        *status |= of_rows;
    }
    return cudaSuccess;
}

cudaError_t dropout(const DropoutArgs &a)
{
    const bool spread = a.dim % 8 != 0 || !in_units(a.x, a.x_stride, a.dtype) || !in_units(a.out, a.out_stride, a.dtype);
    DropoutParams p{};
    p.x = a.x;
    p.out = a.out;
    p.x_stride = a.x_stride;
    p.out_stride = a.out_stride;
    p.n = a.n;
    p.dim = uint32_t(a.dim);
    p.units = uint32_t((a.dim + 7) / 8);
    p.across_log = 8;
    while (p.across_log > (spread ? 5u : 3u) && 1u << p.across_log >= p.units) p.across_log--;      // so that most threads have two units
    p.drop = drop_of(a.drop);
    // 16 bits: as many blocks as fit at once, which take rows in turn; 32 bits: blocks of a row or few, as the hardware deals them out
    // (16384 x 4096: bf16 45.5 us and 48.6 the other way, fp32 79.6 and 90.9, B200)
    const uint32_t down = kThreads >> p.across_log, wide = (p.units + (2u << p.across_log) - 1) / (2u << p.across_log);
    const size_t tall = (a.n + down - 1) / down, most = a.dtype == RD_FP32 ? 65536 : (kSms * kDropoutBlocks + wide - 1) / wide;
    const dim3 grid(unsigned(tall < most ? tall : most), wide);
    auto run = [&](auto T) {
        using Type = decltype(T);
        return spread ? launch(rd_dropout_kernel<Type, true>, grid, kThreads, a.stream, p) : launch(rd_dropout_kernel<Type, false>, grid, kThreads, a.stream, p);
    };
    return a.dtype == RD_FP32 ? run(F32()) : a.dtype == RD_BF16 ? run(B16()) : run(H16());
}

}  // namespace rd
