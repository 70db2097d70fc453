// sm_100a kernels of the root-mean-square norm and of its gradient, for rows of one type: RD_NORM_ROWS is F32, B16 or H16 (a file that
// includes this one each).  The formulas, and what bounds the kernels: rd_norm.cu.
#include "rd_norm_rows.h"

namespace rd {

namespace {

// What a kernel does besides: constants where a branch in its loops would cost, the call's otherwise (kAsk).  kFull: every thread has NV
// units, as for rows of a multiple of 512 or 1024 columns; nothing is asked unit by unit then (gradient of 16384 x 4096 bf16 with dropout
// 120.5 / 114.3 us, B200).
enum Mode { kPlain = 0, kDrop = 1, kEight = 2, kAsk = 4, kFull = 8 };

// What takes a row's largest value (`most` before rstd, `largest` after) to 448.  Very small ones are taken near 1 first (by `lift`), so that
// no quotient overflows.  A largest value that is NaN (a NaN in the row, or an infinity beside its rstd of 0) makes every value NaN.
__device__ __forceinline__ float eighth_factor(float most, float largest, float &lift)
{
    lift = most < 0x1p-60f ? 0x1p64f : 1.0f;
    return isnan(largest) ? largest : most > 0.0f ? 448.0f / (most * lift) : 0.0f;
}

// T: x and out, R: residual and sum, W: the weight.  A thread holds NV units of a row; what it has no unit for is zeros.
template <class T, class R, class W, bool SPREAD, int NV, bool WARP, int MODE> __global__ void __launch_bounds__(kThreads, SPREAD && NV == 4 ? 2 : 3) rd_norm_kernel(const __grid_constant__ NormParams p)
{
    using UnitT = Unit<T, SPREAD>;
    using UnitR = Unit<R, SPREAD>;
    constexpr uint32_t kT = UnitT::bytes / 8, kR = UnitR::bytes / 8;
    const bool drops = MODE & kAsk ? p.drop.border != 0 : bool(MODE & kDrop), eight = MODE & kAsk ? p.out8 : bool(MODE & kEight);
    __shared__ Meeting meeting;
    __shared__ uint4 bits[SPREAD ? kWarps : 1][32];
    __shared__ uint64_t bars[WARP ? kWarps : 1][kMostStages];
    Stream<WARP> stream(bars, SPREAD ? RowRing{0, 0} : p.ring);
    pdl_wait();
    if (p.release_early) pdl_release();
    if (!WARP) cluster_begins(p.blocks);
    const Place<SPREAD, WARP, bool(MODE & kFull)> at(p.units, p.per_block, p.blocks, p.threads, gridDim.x);
    const uint32_t unit0 = WARP ? 0 : at.rank * p.per_block, own = at.end - unit0;
    const Piece pieces[2] = {{p.x, p.x_stride * kT, UnitT::bytes}, {p.residual, p.residual_stride * kR, UnitR::bytes}};
    if (!SPREAD && stream.asks)
        for (uint32_t i = 0; i < stream.stages && at.row + i * at.rows < p.n; i++) stream.ask(i, pieces, at.row + i * at.rows, unit0, own);
    if (!WARP) cluster_has_begun(p.blocks);
    uint32_t turn = 0;
    for (size_t row = at.row; row < p.n; row += at.rows, turn++) {
        UnitT x[NV];
        UnitR res[NV];
        const void *x_row, *res_row;
        if (SPREAD) {
            x_row = at_byte(p.x, row * p.x_stride * kT);
            res_row = at_byte(p.residual, row * p.residual_stride * kR);
        } else {
            const unsigned char *here = stream.wait();
            x_row = here - unit0 * UnitT::bytes;
            res_row = here + own * UnitT::bytes - unit0 * UnitR::bytes;
        }
#pragma unroll
        for (int k = 0; k < NV; k++) {
            x[k].template load<!SPREAD>(x_row, at.unit + k * at.step, p.dim, at.has(k));
            res[k].template load<!SPREAD>(res_row, at.unit + k * at.step, p.dim, at.has(k) && p.residual);
        }
        void *const sum_row = at_byte(p.sum, row * p.sum_stride * kR);
        Pair s[NV][4], squares = 0;
        float2 stat = make_float2(0.0f, 0.0f);        // sum of squares, largest |s w|
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const uint32_t unit = at.unit + k * at.step;
            x[k].get(s[k]);
            if (drops) drop_values<SPREAD>(p.drop, bits[SPREAD ? threadIdx.x >> 5 : 0], unit, uint32_t(row), s[k]);
            Pair r[4], w[4];
            res[k].get(r);
#pragma unroll
            for (int i = 0; i < 4; i++) s[k][i] = add2(s[k][i], r[i]);
            if (p.sum && at.has(k)) {
                UnitR o;
                o.set(s[k]);
                o.store(sum_row, unit, p.dim);
            }
            Unit<W, SPREAD> weight;
            weight.load(p.weight, unit, p.dim, at.has(k));
            weight.get(w);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                squares = fma2(s[k][i], s[k][i], squares);
                s[k][i] = mul2(s[k][i], w[i]);
            }
            if (eight)
#pragma unroll
                for (int i = 0; i < 4; i++) stat.y = most_of(stat.y, both(s[k][i]));
        }
        const float2 sums = both(squares);
        stat.x = sums.x + sums.y;
        stat = join_row<WARP>(stat, eight, meeting, turn, p.blocks, at.rank);
        if (!SPREAD) {
            // everyone has read this row
            const size_t later = row + stream.stages * at.rows;
            if (stream.asks && later < p.n && !stream.dead) stream.ask(stream.s, pieces, later, unit0, own);
            stream.advance();
        }
        const float rstd = rsqrtf(fmaf(stat.x, p.inv_dim, p.eps));
        const float largest = stat.y * rstd;
        float factor = rstd;
        if (eight) {
            float lift;
            factor = eighth_factor(stat.y, largest, lift);
            if (lift != 1.0f) {
#pragma unroll
                for (int k = 0; k < NV; k++)
#pragma unroll
                    for (int i = 0; i < 4; i++) s[k][i] = mul2(s[k][i], pair(lift, lift));
            }
        }
        if (at.first()) {
            if (p.rstd) p.rstd[row] = rstd;
            if (eight) p.out_scale[row] = largest / 448.0f;
        }
        const Pair factors = pair(factor, factor);
        void *const out_row = at_byte(p.out, row * p.out_stride * (eight ? 1 : kT));
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const uint32_t unit = at.unit + k * at.step;
#pragma unroll
            for (int i = 0; i < 4; i++) s[k][i] = mul2(s[k][i], factors);
            if (eight) {
                uint8_t *out = static_cast<uint8_t *>(out_row);
                uint32_t q[4];
#pragma unroll
                for (int i = 0; i < 4; i++) q[i] = __nv_cvt_float2_to_fp8x2(both(s[k][i]), __NV_SATFINITE, __NV_E4M3);
                if constexpr (!SPREAD) {
                    if (at.has(k)) *reinterpret_cast<uint2 *>(out + unit * 8) = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        if (at.has(k) && column_of<true>(unit, i) < p.dim) out[column_of<true>(unit, i)] = uint8_t(i & 1 ? q[i / 2] >> 8 : q[i / 2]);
                }
            } else if (at.has(k)) {
                UnitT o;
                o.set(s[k]);
                o.store(out_row, unit, p.dim);
            }
        }
    }
    if (!p.release_early) pdl_release();
    if (stream.dead) drain();
}

// Rows of at most 32 units, as of a head: LANES lanes (8, 16 or 32) have one, so that a warp has four, two or one at a time; a lane has a
// unit, the next row's operands on their way, and the weight for good.
template <class T, class R, class W, int LANES> __global__ void __launch_bounds__(kThreads, kShortBlocks) rd_norm_short_kernel(const __grid_constant__ NormParams p)
{
    using UnitT = Unit<T, false>;
    using UnitR = Unit<R, false>;
    constexpr uint32_t kT = UnitT::bytes / 8, kR = UnitR::bytes / 8, kRows = 32 / LANES;
    pdl_wait();
    if (p.release_early) pdl_release();
    const uint32_t lane = threadIdx.x & 31, unit = lane % LANES;
    const bool mine = unit < p.units;
    const size_t step = size_t(gridDim.x) * kWarps * kRows;
    size_t base = (size_t(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * kRows;          // the warp's first row
    UnitT x;
    UnitR res;
    Unit<W, false> weight;
    Pair w[4];
    auto load = [&](size_t row) {
        x.load(at_byte(p.x, row * p.x_stride * kT), unit, p.dim, mine && row < p.n);
        res.load(at_byte(p.residual, row * p.residual_stride * kR), unit, p.dim, mine && row < p.n && p.residual);
    };
    weight.load(p.weight, unit, p.dim, mine);
    weight.get(w);
    load(base + lane / LANES);
    for (; base < p.n; base += step) {
        const size_t row = base + lane / LANES;
        const bool live = mine && row < p.n;
        Pair s[4], r[4];
        x.get(s);
        res.get(r);
        load(row + step);
        if (p.drop.border) drop_values<false>(p.drop, nullptr, unit, uint32_t(row), s);
#pragma unroll
        for (int i = 0; i < 4; i++) s[i] = add2(s[i], r[i]);
        if (p.sum && live) {
            UnitR o;
            o.set(s);
            o.store(at_byte(p.sum, row * p.sum_stride * kR), unit, p.dim);
        }
        Pair squares = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            squares = fma2(s[i], s[i], squares);
            s[i] = mul2(s[i], w[i]);
        }
        float sum = both(squares).x + both(squares).y, most = 0.0f;
#pragma unroll
        for (int d = LANES / 2; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (p.out8) {
#pragma unroll
            for (int i = 0; i < 4; i++) most = most_of(most, both(s[i]));
#pragma unroll
            for (int d = LANES / 2; d; d /= 2) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, d));
        }
        const float rstd = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
        const float largest = most * rstd;
        float lift = 1.0f;
        const float factor = p.out8 ? eighth_factor(most, largest, lift) : rstd;
        if (unit == 0 && live) {
            if (p.rstd) p.rstd[row] = rstd;
            if (p.out8) p.out_scale[row] = largest / 448.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; i++) s[i] = mul2(lift != 1.0f ? mul2(s[i], pair(lift, lift)) : s[i], pair(factor, factor));
        if (!live) continue;
        if (p.out8) {
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; i++) q[i] = __nv_cvt_float2_to_fp8x2(both(s[i]), __NV_SATFINITE, __NV_E4M3);
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.out) + row * p.out_stride + unit * 8) = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
        } else {
            UnitT o;
            o.set(s);
            o.store(at_byte(p.out, row * p.out_stride * kT), unit, p.dim);
        }
    }
    if (!p.release_early) pdl_release();
}

// ------------------------------------------------------------------------------------------------ gradient

template <class T> __device__ __forceinline__ float element(const void *p, size_t at)
{
    if constexpr (std::is_same_v<T, F32>) return static_cast<const float *>(p)[at];
    else if constexpr (std::is_same_v<T, B16>) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[at]);
    else return __half2float(static_cast<const __half *>(p)[at]);
}

// grad_weight of 16 columns over all rows, by one block: for few rows, where another launch would cost more than reading twice.
template <class T, class R, class W> __device__ __forceinline__ void sum_columns(const NormGradParams &p, float (*sums)[kSumColumns])
{
    const uint32_t x = threadIdx.x % kSumColumns, y = threadIdx.x / kSumColumns, down = blockDim.x / kSumColumns, column = (blockIdx.x - p.row_blocks) * kSumColumns + x;
    float v = 0.0f;
    if (column < p.dim)
#pragma unroll 8
        for (uint32_t row = y; row < uint32_t(p.n); row += down)
            v = fmaf(element<T>(p.grad_out, row * p.grad_out_stride + column) * element<R>(p.sum, row * p.sum_stride + column), p.rstd[row], v);
    sums[y][x] = v;
    __syncthreads();
    if (y || column >= p.dim) return;
    for (uint32_t k = 1; k < down; k++) v += sums[k][x];
    if constexpr (std::is_same_v<W, F32>) static_cast<float *>(p.grad_weight)[column] = v;
    else if constexpr (std::is_same_v<W, B16>) static_cast<__nv_bfloat16 *>(p.grad_weight)[column] = __float2bfloat16_rn(v);
    else static_cast<__half *>(p.grad_weight)[column] = __float2half_rn(v);
}

// Persistent groups of threads that take rows in turn; a thread's columns stay the same, so that grad_weight adds up in its registers.
// With the sum over a row of grad_out w s = m:  grad = r (grad_out w - s (r^2 m / dim)) + grad_sum.
template <class T, class R, class W, bool SPREAD, int NV, bool WARP, int MODE>
__global__ void __launch_bounds__(kThreads, SPREAD && NV == 4 ? 2 : 3) rd_norm_grad_kernel(const __grid_constant__ NormGradParams p)
{
    using UnitT = Unit<T, SPREAD>;
    using UnitR = Unit<R, SPREAD>;
    constexpr uint32_t kT = UnitT::bytes / 8, kR = UnitR::bytes / 8;
    const bool drops = MODE & kAsk ? p.drop.border != 0 : bool(MODE & kDrop);
    __shared__ float column_sums[kThreads / kSumColumns][kSumColumns];
    __shared__ Meeting meeting;
    __shared__ uint4 bits[SPREAD ? kWarps : 1][32];
    __shared__ uint64_t bars[WARP ? kWarps : 1][kMostStages];
    Stream<WARP> stream(bars, SPREAD ? RowRing{0, 0} : p.ring);
    pdl_wait();
    if (p.release_early) pdl_release();
    if (blockIdx.x >= p.row_blocks) {
        sum_columns<T, R, W>(p, column_sums);
        return;                       // whole clusters of them
    }
    if (!WARP) cluster_begins(p.blocks);
    const Place<SPREAD, WARP, bool(MODE & kFull)> at(p.units, p.per_block, p.blocks, p.threads, p.row_blocks);
    const uint32_t unit0 = WARP ? 0 : at.rank * p.per_block, own = at.end - unit0;
    const Piece pieces[3] = {{p.grad_out, p.grad_out_stride * kT, UnitT::bytes}, {p.sum, p.sum_stride * kR, UnitR::bytes}, {p.grad_sum, p.grad_sum_stride * kR, UnitR::bytes}};
    if (!SPREAD && stream.asks)
        for (uint32_t i = 0; i < stream.stages && at.row + i * at.rows < p.n; i++) stream.ask(i, pieces, at.row + i * at.rows, unit0, own);
    Pair acc[NV][4] = {};
    uint32_t turn = 0;
    float next_rstd = at.row < p.n ? p.rstd[at.row] : 0.0f;
    if (!WARP) cluster_has_begun(p.blocks);
    for (size_t row = at.row; row < p.n; row += at.rows, turn++) {
        const float rstd = next_rstd;
        if (row + at.rows < p.n) next_rstd = p.rstd[row + at.rows];
        const Pair rstds = pair(rstd, rstd);
        const void *up_row, *sum_row, *more_row;
        if (SPREAD) {
            up_row = at_byte(p.grad_out, row * p.grad_out_stride * kT);
            sum_row = at_byte(p.sum, row * p.sum_stride * kR);
            more_row = at_byte(p.grad_sum, row * p.grad_sum_stride * kR);
        } else {
            const unsigned char *here = stream.wait();
            up_row = here - unit0 * UnitT::bytes;
            sum_row = here + own * UnitT::bytes - unit0 * UnitR::bytes;
            more_row = here + own * (UnitT::bytes + UnitR::bytes) - unit0 * UnitR::bytes;
        }
        // from the ring every operand is read where it is needed, twice; otherwise once, ahead
        UnitT up[NV];
        UnitR sum[NV], more[NV];
        auto load = [&](int k) {
            up[k].template load<!SPREAD>(up_row, at.unit + k * at.step, p.dim, at.has(k));
            sum[k].template load<!SPREAD>(sum_row, at.unit + k * at.step, p.dim, at.has(k));
        };
        auto load_more = [&](int k) { more[k].template load<!SPREAD>(more_row, at.unit + k * at.step, p.dim, at.has(k) && p.grad_sum); };
        if (SPREAD) {
#pragma unroll
            for (int k = 0; k < NV; k++) {
                load(k);
                load_more(k);
            }
        }
        Pair dots = 0;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            if (!SPREAD) load(k);
            Pair u[4], s[4], w[4];
            up[k].get(u);
            sum[k].get(s);
            Unit<W, SPREAD> weight;
            weight.load(p.weight, at.unit + k * at.step, p.dim, at.has(k));
            weight.get(w);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const Pair y = mul2(u[i], s[i]);
                acc[k][i] = fma2(y, rstds, acc[k][i]);
                dots = fma2(y, w[i], dots);
            }
        }
        const float2 dot = both(dots);
        const float slope = join_row<WARP>(make_float2(dot.x + dot.y, 0.0f), false, meeting, turn, p.blocks, at.rank).x * p.inv_dim * rstd * rstd;
        const Pair slopes = pair(-slope, -slope);
        if (!SPREAD) {
            // everyone is through with the row before this one
            const size_t later = row + (stream.stages - 1) * at.rows;
            if (stream.asks && turn > 0 && later < p.n && !stream.dead) stream.ask(stream.s == 0 ? stream.stages - 1 : stream.s - 1, pieces, later, unit0, own);
            stream.advance();
        }
        if (!p.want_rows) continue;
        void *const gr_row = at_byte(p.grad_residual, row * p.grad_residual_stride * kR), *const gx_row = at_byte(p.grad_x, row * p.grad_x_stride * kT);
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const uint32_t unit = at.unit + k * at.step;
            if (!SPREAD) {
                load(k);
                load_more(k);
            }
            Pair u[4], s[4], w[4];
            up[k].get(u);
            sum[k].get(s);
            Unit<W, SPREAD> weight;
            weight.load(p.weight, unit, p.dim, at.has(k));
            weight.get(w);
#pragma unroll
            for (int i = 0; i < 4; i++) u[i] = fma2(slopes, s[i], mul2(u[i], w[i]));
            more[k].get(s);
#pragma unroll
            for (int i = 0; i < 4; i++) u[i] = fma2(rstds, u[i], s[i]);
            if (p.grad_residual && at.has(k)) {
                UnitR o;
                o.set(u);
                o.store(gr_row, unit, p.dim);
            }
            if (p.grad_x) {
                if (drops) drop_values<SPREAD>(p.drop, bits[SPREAD ? threadIdx.x >> 5 : 0], unit, uint32_t(row), u);
                if (at.has(k)) {
                    UnitT o;
                    o.set(u);
                    o.store(gx_row, unit, p.dim);
                }
            }
        }
    }
    if (!p.release_early) pdl_release();
    if (stream.dead) drain();
    if (!p.part) return;
    if constexpr (WARP) {
        // the block's warps, one after the other in shared memory (the ring's, which no copy is on its way to), in order
        float *of_warp = reinterpret_cast<float *>(ring);
        const uint32_t warp = threadIdx.x >> 5;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.has(k))
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const uint32_t j = column_of<SPREAD>(at.unit + k * at.step, i);
                    if (!SPREAD || j < p.dim) of_warp[warp * p.dim + j] = i & 1 ? both(acc[k][i / 2]).y : both(acc[k][i / 2]).x;
                }
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < p.dim; j += kThreads) {
            float v = of_warp[j];
#pragma unroll
            for (int k = 1; k < kWarps; k++) v += of_warp[k * p.dim + j];
            p.part[size_t(blockIdx.x) * p.dim + j] = v;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.has(k)) {
                Unit<F32, SPREAD> o;
                o.set(acc[k]);
                o.store(p.part + at.row * p.dim, at.unit + k * at.step, p.dim);
            }
    }
}

// The same for the gradient.
template <class T, class R, class W, int LANES> __global__ void __launch_bounds__(kThreads, kShortBlocks) rd_norm_grad_short_kernel(const __grid_constant__ NormGradParams p)
{
    using UnitT = Unit<T, false>;
    using UnitR = Unit<R, false>;
    constexpr uint32_t kT = UnitT::bytes / 8, kR = UnitR::bytes / 8, kRows = 32 / LANES;
    __shared__ float column_sums[kThreads / kSumColumns][kSumColumns];
    __shared__ float of_row[kWarps * kRows][LANES * 8];
    pdl_wait();
    if (p.release_early) pdl_release();
    if (blockIdx.x >= p.row_blocks) {
        sum_columns<T, R, W>(p, column_sums);
        return;
    }
    const uint32_t lane = threadIdx.x & 31, unit = lane % LANES, place = (threadIdx.x >> 5) * kRows + lane / LANES;
    const bool mine = unit < p.units;
    const size_t step = size_t(p.row_blocks) * kWarps * kRows;
    size_t base = (size_t(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * kRows;          // the warp's first row
    UnitT up;
    UnitR sum, more;
    Unit<W, false> weight;
    float rstd;
    Pair w[4], acc[4] = {};
    auto load = [&](size_t row) {
        const bool live = mine && row < p.n;
        up.load(at_byte(p.grad_out, row * p.grad_out_stride * kT), unit, p.dim, live);
        sum.load(at_byte(p.sum, row * p.sum_stride * kR), unit, p.dim, live);
        more.load(at_byte(p.grad_sum, row * p.grad_sum_stride * kR), unit, p.dim, live && p.grad_sum);
        rstd = live ? p.rstd[row] : 0.0f;
    };
    weight.load(p.weight, unit, p.dim, mine);
    weight.get(w);
    load(base + lane / LANES);
    for (; base < p.n; base += step) {
        const size_t row = base + lane / LANES;
        const bool live = mine && row < p.n;
        Pair u[4], s[4], m[4], dots = 0;
        up.get(u);
        sum.get(s);
        more.get(m);
        const float r = rstd;
        load(row + step);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const Pair y = mul2(u[i], s[i]);
            acc[i] = fma2(y, pair(r, r), acc[i]);
            dots = fma2(y, w[i], dots);
        }
        float dot = both(dots).x + both(dots).y;
#pragma unroll
        for (int d = LANES / 2; d; d /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, d);
        if (!live || !p.want_rows) continue;
        const float slope = dot * p.inv_dim * r * r;
#pragma unroll
        for (int i = 0; i < 4; i++) u[i] = fma2(pair(r, r), fma2(pair(-slope, -slope), s[i], mul2(u[i], w[i])), m[i]);
        if (p.grad_residual) {
            UnitR o;
            o.set(u);
            o.store(at_byte(p.grad_residual, row * p.grad_residual_stride * kR), unit, p.dim);
        }
        if (p.grad_x) {
            if (p.drop.border) drop_values<false>(p.drop, nullptr, unit, uint32_t(row), u);
            UnitT o;
            o.set(u);
            o.store(at_byte(p.grad_x, row * p.grad_x_stride * kT), unit, p.dim);
        }
    }
    if (!p.release_early) pdl_release();
    if (!p.part) return;
    if (mine)
#pragma unroll
        for (int i = 0; i < 4; i++) of_row[place][unit * 8 + 2 * i] = both(acc[i]).x, of_row[place][unit * 8 + 2 * i + 1] = both(acc[i]).y;
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < p.dim; j += kThreads) {
        float v = of_row[0][j];
#pragma unroll
        for (int k = 1; k < int(kWarps * kRows); k++) v += of_row[k][j];
        p.part[size_t(blockIdx.x) * p.dim + j] = v;
    }
}

// ------------------------------------------------------------------------------------------------ launches

template <auto KERNEL, typename P> cudaError_t launch_rows(const P &p, const RowShape &s, const RowDeal &d, cudaStream_t stream, size_t more_blocks = 0)
{
    if (s.smem > 0) {
        static std::atomic<bool> ready[64];
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        if (e == cudaSuccess && (device >= 64 || !ready[device].load(std::memory_order_acquire))) {
            e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kRingBytes));
            if (e == cudaSuccess && device < 64) ready[device].store(true, std::memory_order_release);
        }
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(unsigned(s.groups * d.blocks + more_blocks));
    c.blockDim = dim3(d.threads);
    c.dynamicSmemBytes = s.smem;
    c.stream = stream;
    cudaLaunchAttribute attrs[2] = {pdl_attribute()};
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = d.blocks;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    c.attrs = attrs;
    c.numAttrs = d.blocks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&c, KERNEL, p);
}

template <int N> using Constant = std::integral_constant<int, N>;

// Calls f with the kernel's template arguments: how the row lies, the types of residual and weight.
template <bool GRADIENT, class F> cudaError_t with_shape(bool spread, const RowDeal &d, F &&f)
{
    using std::integral_constant;
    using Yes = integral_constant<bool, true>;
    using No = integral_constant<bool, false>;
    using Two = integral_constant<int, 2>;
    using Four = integral_constant<int, 4>;
    if (spread && d.warp) return f(Yes(), Two(), Yes());
    if (spread) return d.nv == 2 ? f(Yes(), Two(), No()) : f(Yes(), Four(), No());
    if (d.warp) return d.nv == 2 ? f(No(), Two(), Yes()) : f(No(), Four(), Yes());
    if constexpr (GRADIENT)
        if (d.nv == 2) return f(No(), Two(), No());
    return f(No(), Four(), No());
}
template <class F> cudaError_t with_lanes(int lanes, F &&f) { return lanes == 8 ? f(Constant<8>()) : lanes == 16 ? f(Constant<16>()) : f(Constant<32>()); }
template <class T, class F> cudaError_t with_types(int sum_dtype, int weight_dtype, F &&f)
{
    if constexpr (std::is_same_v<T, F32>) return f(F32(), F32());
    else if (sum_dtype == RD_FP32) return weight_dtype == RD_FP32 ? f(F32(), F32()) : f(F32(), T());
    else return weight_dtype == RD_FP32 ? f(T(), F32()) : f(T(), T());
}

}  // namespace

template <> cudaError_t launch_norm<RD_NORM_ROWS>(const NormParams &p, const NormCall &c)
{
    using T = RD_NORM_ROWS;
    if (c.deal.lanes)
        return with_types<T>(c.sum_dtype, c.weight_dtype, [&](auto R, auto W) {
            using RT = decltype(R);
            using WT = decltype(W);
            return with_lanes(c.deal.lanes, [&](auto LANES) { return launch_rows<rd_norm_short_kernel<T, RT, WT, LANES()>>(p, c.shape, c.deal, c.stream); });
        });
    return with_shape<false>(c.spread, c.deal, [&](auto SPREAD, auto NV, auto WARP) {
        return with_types<T>(c.sum_dtype, c.weight_dtype, [&](auto R, auto W) {
            using RT = decltype(R);
            using WT = decltype(W);
            if constexpr (SPREAD()) {
                return launch_rows<rd_norm_kernel<T, RT, WT, true, NV(), WARP(), kAsk>>(p, c.shape, c.deal, c.stream);
            } else {
                auto run = [&](auto MODE) { return launch_rows<rd_norm_kernel<T, RT, WT, false, NV(), WARP(), MODE()>>(p, c.shape, c.deal, c.stream); };
                if (p.out8 && p.drop.border) return run(Constant<kDrop | kEight>());
                if (p.out8) return c.deal.full() ? run(Constant<kEight | kFull>()) : run(Constant<kEight>());
                // (with the random bits of four units at once registers run out: 16384 x 4096 bf16 89 us, kFull 97)
                if (p.drop.border) return run(Constant<kDrop>());
                return c.deal.full() ? run(Constant<kPlain | kFull>()) : run(Constant<kPlain>());
            }
        });
    });
}

template <> cudaError_t launch_norm_grad<RD_NORM_ROWS>(const NormGradParams &p, const NormCall &c)
{
    using T = RD_NORM_ROWS;
    if (c.deal.lanes)
        return with_types<T>(c.sum_dtype, c.weight_dtype, [&](auto R, auto W) {
            using RT = decltype(R);
            using WT = decltype(W);
            return with_lanes(c.deal.lanes, [&](auto LANES) { return launch_rows<rd_norm_grad_short_kernel<T, RT, WT, LANES()>>(p, c.shape, c.deal, c.stream, c.more_blocks); });
        });
    return with_shape<true>(c.spread, c.deal, [&](auto SPREAD, auto NV, auto WARP) {
        return with_types<T>(c.sum_dtype, c.weight_dtype, [&](auto R, auto W) {
            using RT = decltype(R);
            using WT = decltype(W);
            if constexpr (SPREAD()) {
                return launch_rows<rd_norm_grad_kernel<T, RT, WT, true, NV(), WARP(), kAsk>>(p, c.shape, c.deal, c.stream, c.more_blocks);
            } else {
                auto run = [&](auto MODE) { return launch_rows<rd_norm_grad_kernel<T, RT, WT, false, NV(), WARP(), MODE()>>(p, c.shape, c.deal, c.stream, c.more_blocks); };
                if (p.drop.border) return c.deal.full() ? run(Constant<kDrop | kFull>()) : run(Constant<kDrop>());
                return c.deal.full() ? run(Constant<kPlain | kFull>()) : run(Constant<kPlain>());
            }
        });
    });
}

template <> cudaError_t norm_rows_status<RD_NORM_ROWS>(int *status)
{
    cudaError_t e = cudaMemcpyFromSymbol(status, g_wait_status, sizeof(int));
    if (e != cudaSuccess) return e;
    const int zero = 0;
    if (*status) e = cudaMemcpyToSymbol(g_wait_status, &zero, sizeof(int));
    return e;
}

}  // namespace rd
