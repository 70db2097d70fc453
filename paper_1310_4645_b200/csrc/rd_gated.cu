// sm_100a kernels of the gated projections of a feed-forward block and of their gradient.
//
//   gate = x Wgᵀ,  up = x Wuᵀ,  out = act(gate) up                          (8 bits: each product times its row's and its column's scale)
//   dgate = dout up act'(gate),  dup = dout act(gate):   dx = dgate Wg + dup Wu,  dWg = dgateᵀ x,  dWu = dupᵀ x
//
// act is g σ(k(g)): silu with k = g, the tanh form of gelu (Hendrycks and Gimpel, 2016) with k = 2 sqrt(2/π) (g + 0.044715 g³), as
// (1 + tanh(k/2)) / 2 = σ(k); or max(g, 0).
//
// Forward: one kernel.  A thread block, or a pair of them, computes tiles of 128 (256) rows by w columns of both projections at once: the
// right operand is w rows of Wg followed by the same w rows of Wu, so that a value's gate and up lie in one lane of tensor memory and
// their product never leaves the thread.  Of a pair one block brings in Wg's rows, the other Wu's.
// Gradient: a pass over gate, up and dout leaves dgate and dup side by side, rounded to 16 bits (the operand type of the products), then
// one launch has both kinds of products, dx over the two widths in one sum, dWg and dWu over the tokens.  Where there are few tiles the sums
// are cut into parts in 32 bits, which a last launch adds up in order.
//
// Operands come in by TMA into a ring of stages of 128 bytes of the summed index; one warp per operand issues the copies, one the
// products, eight take the results; two sets of accumulators, so that one is read while the next is computed.
// What bounds it (B200): many rows, the tensor cores (2048 x 4096 x 12288 bf16: busy 94 % of the active cycles, gradients 97 %) at the clock that
// the board's power limit leaves: 8192 x 4096 x 12288 1.2 to 1.29 ms with gate and up kept = 1.28 to 1.37 PFLOP/s, gradients 2.7 to 3.05; 4096 rows
// in 8 bits 0.31 to 0.39 = 2.1 to 2.6.  Up to some 128 rows, the memory: 36 to 41 us for the weights' 201 MB.  Rows of at most some 256 values, taking
// the results out: 4096 x 64 x 12288 52 us.
#include "rd_block.h"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "rd.h"
#include "rd_launch.h"
#include "rd_mma.h"
#include "rd_ptx.h"
#include "rd_ring.h"

namespace rd {

namespace {

constexpr int kMmaThreads = 128 + 32 * kEpilogueWarps;
constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kTileOverhead = 2;     // what a tile costs besides its products, in steps of the summed index
constexpr size_t kSms = 148;

// ------------------------------------------------------------------------------------------------ activations

__device__ __forceinline__ float reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <int ACT> __device__ __forceinline__ float sigmoid_of(float g)
{
    constexpr float c = 1.5957691216057308f;          // 2 sqrt(2 / pi)
    const float k = ACT == RD_SILU ? g : c * g * fmaf(0.044715f * g, g, 1.0f);
    // ex2 and rcp are within 2^-22; results are rounded to 16 bits
    return reciprocal(1.0f + exp2_fast(-k * kLog2e));
}
template <int ACT> __device__ __forceinline__ float act_value(float g)
{
    if (ACT == RD_RELU) return g < 0.0f ? 0.0f : g;
    return g * sigmoid_of<ACT>(g);
}
template <int ACT> __device__ __forceinline__ void act_both(float g, float &value, float &slope)
{
    if (ACT == RD_RELU) {
        value = g < 0.0f ? 0.0f : g;
        slope = g > 0.0f ? 1.0f : 0.0f;
        return;
    }
    constexpr float c = 1.5957691216057308f;
    const float s = sigmoid_of<ACT>(g), t = s * (1.0f - s), dk = ACT == RD_SILU ? 1.0f : c * fmaf(3.0f * 0.044715f * g, g, 1.0f);
    value = g * s;
    slope = t != 0.0f ? fmaf(g * dk, t, s) : s;       // far out t vanishes before g k'(g) overflows
}
// Calls f with the activation as a constant.
template <class F> __device__ __forceinline__ void with_act(int act, F &&f)
{
    if (act == RD_SILU) f(std::integral_constant<int, RD_SILU>());
    else if (act == RD_GELU) f(std::integral_constant<int, RD_GELU>());
    else f(std::integral_constant<int, RD_RELU>());
}

__device__ __forceinline__ uint32_t pack2(bool bf16, float lo, float hi) { return bf16 ? pack2<true>(lo, hi) : pack2<false>(lo, hi); }
__device__ __forceinline__ float2 widen2(bool bf16, uint32_t v)
{
    if (bf16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}

// ------------------------------------------------------------------------------------------------ the products

struct Out {
    uint16_t *p;              // null: not wanted
    size_t stride;
    int units;                // elements that an access may take: 8, 2 or 1
};
// 16 columns of a warp's 32 rows from column `col` on, of which there are `left`; a lane has a row's.  Where rows do not begin on 16-byte
// boundaries the values change places in 1 KB of shared memory, so that a store has few rows: 4096 x 2048 x 8191 bf16 404 us
// with a lane's values stored by itself, 217 so; gate and up kept 974 and 276 (B200).
__device__ __forceinline__ void put16(const Out &o, uint32_t stage, uint32_t row0, uint32_t rows, uint32_t col, uint32_t left, const uint32_t (&v)[8])
{
    const uint32_t lane = threadIdx.x & 31;
    if (o.units == 8) {
        if (lane >= rows) return;
        uint16_t *dst = o.p + size_t(row0 + lane) * o.stride + col;
        if (left >= 8) reinterpret_cast<uint4 *>(dst)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        if (left >= 16) {
            reinterpret_cast<uint4 *>(dst)[1] = make_uint4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int j = 0; j < 16; j++)
                if (j < left && (j >= 8 || left < 8)) dst[j] = uint16_t(v[j / 2] >> (j & 1 ? 16 : 0));
        }
        return;
    }
    __syncwarp();
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * 32), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * 32 + 16), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    __syncwarp();
    if (o.units == 2) {
#pragma unroll
        for (uint32_t i = 0; i < 8; i++) {
            const uint32_t r = 4 * i + lane / 8, j = lane % 8 * 2;
            uint32_t x;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(stage + r * 32 + j * 2) : "memory");
            uint16_t *dst = o.p + size_t(row0 + r) * o.stride + col + j;
            if (r < rows && j + 1 < left) *reinterpret_cast<uint32_t *>(dst) = x;
            else if (r < rows && j < left) *dst = uint16_t(x);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 16; i++) {
            const uint32_t r = 2 * i + lane / 16, j = lane % 16;
            uint16_t x;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(stage + r * 32 + j * 2) : "memory");
            if (r < rows && j < left) o.p[size_t(row0 + r) * o.stride + col + j] = x;
        }
    }
}

struct alignas(64) GatedParams {
    CUtensorMap a;            // x, boxes of 128 bytes x a_rows
    CUtensorMap gate, up;     // weights, boxes of 128 bytes x tile_w
    uint32_t n, width, steps; // steps: of 128 bytes of the summed index
    uint32_t tile_w;          // columns of a tile, of each projection
    uint32_t stages, stage, a_rows;
    uint32_t staging;         // where in shared memory results change places, 1 KB a warp
    uint32_t group;           // row tiles that go over the width together
    uint32_t idesc;
    int act;
    bool bf16;                // results
    Out out, kept_gate, kept_up;
    const float *x_scale, *gate_scale, *up_scale;
};

struct alignas(64) GradParams {
    CUtensorMap a_k;          // dgate and dup as the left operand of dx, boxes of 64 x a_rows
    CUtensorMap a_mn;         // the same as the transposed left operand of dW, 64 x 64 boxes
    CUtensorMap gate_mn, up_mn;       // weights as the transposed right operand of dx
    CUtensorMap x_mn;         // x as the transposed right operand of dW
    CUtensorMap dx_out, gate_out, up_out;     // results, 64 x 32 boxes
    CUtensorMap dx_parts, dw_parts;           // parts of dx, of dWg and dWu one below the other, in 32 bits, 32 x 32 x 1 boxes
    uint32_t n, dim, width;
    uint32_t half;            // columns of dgate, a multiple of 64: where dup begins
    uint32_t splits, steps_per_split;         // parts that the sum over both widths is cut into for dx, and steps of one
    uint32_t splits_w, steps_per_split_w;     // the same of the sum over rows for dWg and dWu
    uint32_t part_rows;       // rows of a part of dWg: the width, up to whole tiles
    uint32_t a_rows;
    uint32_t idesc;
    uint32_t weights;         // which of dWg (1) and dWu (2) are wanted
    bool want_dx, bf16;
    bool dx_tma, gate_tma, up_tma;            // results that TMA can address
    uint16_t *dx, *dgate, *dup;               // the others, and ends of rows
    size_t dx_stride, dgate_stride, dup_stride;
};

// One unit of work: an output tile and the range of the summed index that goes into it.
struct Work {
    int product;              // 0 gate and up, 1 dx, 2 dW
    uint32_t m0, n0, k0, steps, split;
    bool second;              // dWu
};

// Which units a group of thread blocks (one or a pair, number c of g) gets.
// Forward: bands of p.group row tiles, within a band all row tiles of a column tile one after the other.
template <int CG> struct GatedPlan {
    const GatedParams &p;
    Cursor at;
    uint32_t g, tiles_m, tiles_n, band = 0;
    __device__ __forceinline__ explicit GatedPlan(const GatedParams &params) : p(params), g(gridDim.x / CG)
    {
        tiles_m = (p.n + kRowsM * CG - 1) / (kRowsM * CG);
        tiles_n = (p.width + p.tile_w - 1) / p.tile_w;
        at.set(blockIdx.x / CG, g, min(p.group, tiles_m));
    }
    __device__ __forceinline__ bool next(Work &w)
    {
        while (at.y >= tiles_n) {                          // on to the next band
            const uint32_t over = (at.y - tiles_n) * at.wide + at.x;
            if (++band * p.group >= tiles_m) {
                band--;                                    // stay at the end
                return false;
            }
            at.set(over, g, min(p.group, tiles_m - band * p.group));
        }
        w = Work{0, (band * p.group + at.x) * kRowsM * CG, at.y * p.tile_w, 0, p.steps, 0, false};
        at.advance();
        return true;
    }
};
// How the gradient's units are dealt out over g groups: those of dx first, in turn.  Their number need not divide by g, so the first `more`
// groups get one more of them.  The others then take as many units of dW as that is worth by the steps of the summed index, or come
// first where dW's do not divide either.
struct Deal {
    uint32_t dx_each, more, even;             // units of dx that every group gets; turns of dW that all take part in, the others first
    __host__ __device__ Deal(uint32_t dx_units, uint32_t dx_steps, uint32_t dw_units, uint32_t dw_steps, uint32_t g) : dx_each(dx_units / g), more(dx_units % g)
    {
        const uint32_t worth = more ? (2 * (dx_steps + kTileOverhead) + dw_steps) / (2 * (dw_steps + kTileOverhead)) : 0, ahead = worth * (g - more);
        even = dw_units > ahead ? (dw_units - ahead + g - 1) / g : 0;
    }
};
template <int CG> struct GradPlan {
    static constexpr uint32_t kTileM = kRowsM * CG;
    const GradParams &p;
    Cursor at;
    uint32_t c, g, tiles_n, tiles_m, tiles_w, down, dw_units, left, phase = 0, split = 0, steps_n, steps_w;
    Deal deal;
    __device__ __forceinline__ explicit GradPlan(const GradParams &params)
        : p(params), c(blockIdx.x / CG), g(gridDim.x / CG), tiles_n((p.dim + kTileN - 1) / kTileN), tiles_m((p.n + kTileM - 1) / kTileM), tiles_w((p.width + kTileM - 1) / kTileM),
          down(((p.weights & 1) + (p.weights >> 1)) * tiles_w),              // tiles of dWg and dWu one below the other
          dw_units(down * tiles_n * p.splits_w), steps_n((p.n + kTileK - 1) / kTileK), steps_w(2 * p.half / kTileK),
          deal(p.want_dx ? tiles_m * tiles_n * p.splits : 0, p.steps_per_split, dw_units, p.steps_per_split_w, g)
    {
        left = deal.dx_each + (c < deal.more);
        at.set(c, g, tiles_n);
    }
    __device__ __forceinline__ bool next(Work &w)
    {
        while (left == 0 || (phase != 0 && at.y * tiles_n + at.x >= dw_units)) {
            if (phase == 2) {
                left = 0;
                return false;
            }
            if (++phase == 1) {
                left = deal.even;
                at.set(c < deal.more ? c + g - deal.more : c - deal.more, g, tiles_n);
            } else {
                left = c < deal.more ? 0 : 0xffffffffu;       // until the units run out
                at.set(deal.even * g + c - deal.more, g - deal.more, tiles_n);
            }
        }
        if (phase == 0) {
            while (at.y >= tiles_m) {
                at.y -= tiles_m;
                split++;
            }
            const uint32_t k0 = split * p.steps_per_split;
            w = Work{1, at.y * kTileM, at.x * kTileN, k0 * kTileK, min(p.steps_per_split, steps_w - k0), split, false};
        } else {
            const uint32_t part = p.splits_w == 1 ? 0 : at.y / down, y = at.y - part * down, k0 = part * p.steps_per_split_w;
            const bool second = p.weights == 2 || y >= tiles_w;
            w = Work{2, (y >= tiles_w ? y - tiles_w : y) * kTileM, at.x * kTileN, k0 * kTileK, min(p.steps_per_split_w, steps_n - k0), part, second};
        }
        left--;
        at.advance();
        return true;
    }
};

// A warp has its accumulators in registers: arrives at the first block's barrier.  No release of the cluster's scope: that would wait for
// the results that the warp has stored meanwhile, and nothing in memory is handed over.
template <int CG> __device__ __forceinline__ void accumulators_read(uint32_t bar)
{
    if (CG == 1) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(leader_bar<CG>(bar)) : "memory");
}

template <bool GRADS, int CG> using ShapeOf = Shape<GRADS ? kGrads : kStats, CG>;

template <bool GRADS, bool F8, int CG>
__global__ void __launch_bounds__(kMmaThreads, 1) rd_gated_mma_kernel(const __grid_constant__ std::conditional_t<GRADS, GradParams, GatedParams> p)
{
    using S = ShapeOf<GRADS, CG>;
    uint32_t stages, stage, stage_a;
    if constexpr (GRADS) stages = S::stages, stage = S::stage, stage_a = S::stage_a;
    else stages = p.stages, stage = p.stage, stage_a = p.a_rows * 128;
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
        if constexpr (GRADS) {
            for (const CUtensorMap *map : {&p.a_k, &p.a_mn, &p.gate_mn, &p.up_mn, &p.x_mn}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
        } else {
            for (const CUtensorMap *map : {&p.a, &p.gate, &p.up}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
        }
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

    pdl_start();
    std::conditional_t<GRADS, GradPlan<CG>, GatedPlan<CG>> plan(p);
    bool dead = false;
    Work w;

    if (warp == 0 || warp == 3) {
        // one warp brings in the left operand, another the right one; the copies of both thread blocks and both operands count at
        // the first block's barrier
        const bool elected = elect_one();
        Turn turn(stages);
        const uint32_t lead = leader_bar<CG>(full);
        while (!dead && plan.next(w)) {
            for (uint32_t k = 0; k < w.steps; k++, turn.advance()) {
                const uint32_t a = smem + turn.s * stage, b = a + stage_a, bar = lead + 8 * turn.s;
                if (!warp_wait(empty + 8 * turn.s, turn.parity ^ 1)) { dead = true; break; }
                if (!elected) continue;
                if constexpr (!GRADS) {
                    const uint32_t x = k * (F8 ? 128 : 64);
                    if (warp == 0) {
                        if (rank == 0) bar_expect(full + 8 * turn.s, CG * p.a_rows * 128 + 2 * p.tile_w * 128);
                        tma_load<CG>(a, &p.a, x, w.m0 + rank * kRowsM, bar);
                    } else if (CG == 2) {
                        tma_load<CG>(b, rank ? &p.up : &p.gate, x, w.n0, bar);
                    } else {
                        tma_load<CG>(b, &p.gate, x, w.n0, bar);
                        tma_load<CG>(b + p.tile_w * 128, &p.up, x, w.n0, bar);
                    }
                } else {
                    const uint32_t kk = w.k0 + k * kTileK, m0 = w.m0 + rank * kRowsM, n0 = w.n0 + rank * S::rows_n;
                    if (warp == 0) {
                        if (rank == 0) bar_expect(full + 8 * turn.s, CG * ((w.product == 2 ? S::stage_a : p.a_rows * 128) + S::stage_b));
                        if (w.product == 2) {
#pragma unroll
                            for (int j = 0; j < kRowsM / 64; j++) tma_load<CG>(a + j * 8192, &p.a_mn, (w.second ? p.half : 0) + m0 + 64 * j, kk, bar);
                        } else {
                            tma_load<CG>(a, &p.a_k, kk, m0, bar);
                        }
                    } else {
                        const CUtensorMap *map = w.product == 2 ? &p.x_mn : kk < p.half ? &p.gate_mn : &p.up_mn;
                        const uint32_t y = w.product == 1 && kk >= p.half ? kk - p.half : kk;
#pragma unroll
                        for (int j = 0; j < S::rows_n / 64; j++) tma_load<CG>(b + j * 8192, map, n0 + 64 * j, y, bar);
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
            Turn turn(stages);
            uint32_t tile = 0;
            while (!dead && plan.next(w)) {
                const uint32_t buf = tile & 1;
                if (!warp_wait(acc_empty + 8 * buf, (tile / 2 & 1) ^ 1)) { dead = true; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const bool ta = w.product == 2, tb = w.product != 0;
                const uint32_t idesc = p.idesc | (ta ? 1u << 15 : 0u) | (tb ? 1u << 16 : 0u);
                const uint32_t step_a = ta ? 2048 >> 4 : 32 >> 4, step_b = tb ? 2048 >> 4 : 32 >> 4;
                const uint32_t acc = tmem + buf * kTileN;
                for (uint32_t k = 0; k < w.steps; k++, turn.advance()) {
                    const uint32_t a = smem + turn.s * stage, b = a + stage_a;
                    if (!warp_wait(full + 8 * turn.s, turn.parity)) { dead = true; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = operand(a, ta), db = operand(b, tb);
                    if (elected) {
                        // 32 bytes of the summed index at a time, whatever the type
#pragma unroll
                        for (int j = 0; j < 4; j++) mma<CG, F8>(acc, da + j * step_a, db + j * step_b, idesc, k != 0 || j != 0);
                        mma_commit<CG>(empty + 8 * turn.s);
                    }
                }
                if (!dead && elected) mma_commit<CG>(acc_full + 8 * buf);
                tile++;
            }
            if (dead) drain();
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, half = (warp - 4) >> 2;        // rows 32 * quarter.. of the tile, half of its columns
        uint32_t tile = 0;
        while (plan.next(w)) {
            const uint32_t row0 = w.m0 + rank * kRowsM + 32 * quarter, row = row0 + lane, buf = tile & 1;
            // 8 bits: the row's scale, and those of the warp's up to 64 columns, two a lane, fetched while the products are under way
            float x_scale = 1.0f, gate_scales[2], up_scales[2];
            if constexpr (!GRADS && F8) {
                const uint32_t at = w.n0 + 16 * (half ? ((p.tile_w + 15) / 16 + 1) / 2 : 0) + lane;
                if (row < p.n) x_scale = p.x_scale[row];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const bool there = at + 32 * i < p.width;
                    gate_scales[i] = there ? p.gate_scale[at + 32 * i] : 0.0f;
                    up_scales[i] = there ? p.up_scale[at + 32 * i] : 0.0f;
                }
            }
            if (!warp_wait(acc_full + 8 * buf, tile / 2 & 1)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + buf * kTileN + (uint32_t(32 * quarter) << 16);
            // the accumulators are free for the next tile but one as soon as their last columns are in registers
            auto release = [&]() {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) accumulators_read<CG>(acc_empty + 8 * buf);
            };
            if constexpr (!GRADS) {
                // a tile's columns by 16, half of them each warp's; the last 16 may be 8, and what lies behind them the other projection's
                const uint32_t chunks = (p.tile_w + 15) / 16, first = half ? (chunks + 1) / 2 : 0, last = half ? chunks : (chunks + 1) / 2;
                const uint32_t columns = min(p.tile_w, p.width - w.n0), rows = row0 < p.n ? min(32u, p.n - row0) : 0, stage = smem + p.staging + (warp - 4) * 1024;
                const int count = int(last - first);
                // 16 columns of both are on their way while the 16 before them are worked on
                uint32_t gates[2][16], ups[2][16];
                auto load = [&](int k) {
                    tmem_load(acc + 16 * (first + k), gates[k & 1]);
                    tmem_load(acc + p.tile_w + 16 * (first + k), ups[k & 1]);
                };
                if (count > 0) load(0);
                else release();
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    if (k >= count) break;
                    uint32_t(&g)[16] = gates[k & 1], (&u)[16] = ups[k & 1];
                    tmem_wait(g);
                    tmem_wait(u);
                    if (k + 1 < count) load(k + 1);
                    else release();
                    const uint32_t c = first + k;
                    if (16 * c >= columns) continue;
                    const uint32_t col = w.n0 + 16 * c, left = columns - 16 * c;
                    if (F8) {
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            const int at = (16 * k + j) % 32;
                            // one after the other: the product of two scales may leave fp32's range where the result does not
                            g[j] = __float_as_uint(__uint_as_float(g[j]) * x_scale * __shfl_sync(0xffffffffu, gate_scales[k / 2], at));
                            u[j] = __float_as_uint(__uint_as_float(u[j]) * x_scale * __shfl_sync(0xffffffffu, up_scales[k / 2], at));
                        }
                    }
                    uint32_t o[8];
                    with_act(p.act, [&](auto ACT) {
#pragma unroll
                        for (int j = 0; j < 8; j++)
                            o[j] = pack2(p.bf16, act_value<decltype(ACT)::value>(__uint_as_float(g[2 * j])) * __uint_as_float(u[2 * j]),
                                         act_value<decltype(ACT)::value>(__uint_as_float(g[2 * j + 1])) * __uint_as_float(u[2 * j + 1]));
                    });
                    put16(p.out, stage, row0, rows, col, left, o);
                    if (p.kept_gate.p) {
#pragma unroll
                        for (int j = 0; j < 8; j++) o[j] = pack2(p.bf16, __uint_as_float(g[2 * j]), __uint_as_float(g[2 * j + 1]));
                        put16(p.kept_gate, stage, row0, rows, col, left, o);
                    }
                    if (p.kept_up.p) {
#pragma unroll
                        for (int j = 0; j < 8; j++) o[j] = pack2(p.bf16, __uint_as_float(u[2 * j]), __uint_as_float(u[2 * j + 1]));
                        put16(p.kept_up, stage, row0, rows, col, left, o);
                    }
                    __syncwarp();                // the next load of the accumulators is the whole warp's
                }
            } else {
                const uint32_t box = boxes + (warp - 4) * kBox, col0 = w.n0 + 128 * half;
                const bool parts = (w.product == 1 ? p.splits : p.splits_w) > 1;
                const CUtensorMap *parts_map = w.product == 1 ? &p.dx_parts : &p.dw_parts;
                const uint32_t parts_row = row0 + (w.second ? p.part_rows : 0);
                const CUtensorMap *map = w.product == 1 ? &p.dx_out : w.second ? &p.up_out : &p.gate_out;
                const bool tma = w.product == 1 ? p.dx_tma : w.second ? p.up_tma : p.gate_tma;
                const uint32_t rows = w.product == 1 ? p.n : p.width;
                // 32 columns are on their way while the 32 before them are worked on
                uint32_t v[2][32];
                tmem_load(acc + 128 * half, v[0]);
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    uint32_t(&x)[32] = v[c & 1];
                    tmem_wait(x);
                    if (c < 3) tmem_load(acc + 128 * half + 32 * (c + 1), v[(c + 1) & 1]);
                    else release();
                    const uint32_t col = col0 + 32 * c;
                    if (parts) {
                        box_wait(lane, false);
#pragma unroll
                        for (int q = 0; q < 8; q++) box_put(box, lane, q, x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                        if (box_full(lane, true) && col < p.dim && row0 < rows) {
                            tma_store(parts_map, box, col, parts_row, w.split);
                            box_sent();
                        }
                        continue;
                    }
                    // a box of 64 columns
                    box_wait(lane, c & 1);
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        uint32_t o[4];
#pragma unroll
                        for (int j = 0; j < 4; j++) o[j] = pack2(p.bf16, __uint_as_float(x[8 * q + 2 * j]), __uint_as_float(x[8 * q + 2 * j + 1]));
                        box_put(box, lane, 4 * (c & 1) + q, o[0], o[1], o[2], o[3]);
                    }
                    if (tma && box_within(col - 32 * (c & 1), p.dim)) {
                        if (box_full(lane, c & 1) && col - 32 < p.dim && row0 < rows) {
                            tma_store(map, box, col - 32, row0);
                            box_sent();
                        }
                    } else if (c & 1) {
                        // rows that TMA cannot address, or whose end it would overwrite: the warp writes them one after the other, two
                        // elements a lane
                        __syncwarp();
                        const size_t stride = w.product == 1 ? p.dx_stride : w.second ? p.dup_stride : p.dgate_stride;
                        uint16_t *dst = (w.product == 1 ? p.dx : w.second ? p.dup : p.dgate) + size_t(row0) * stride + (col - 32);
                        const uint32_t here = row0 < rows ? min(32u, rows - row0) : 0;
#pragma unroll 4
                        for (uint32_t r = 0; r < here; r++) {
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const uint32_t j = lane + 32 * i;
                                uint16_t y;
                                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(box + r * 128 + (((j / 8) ^ (r & 7)) * 16) + j % 8 * 2) : "memory");
                                if (col - 32 + j < p.dim) dst[size_t(r) * stride + j] = y;
                            }
                        }
                        __syncwarp();
                    }
                }
            }
            tile++;
        }
        if (GRADS && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    pair_sync<CG>();                             // neither block of a pair leaves while the other may still signal it
    if (warp == 2) {
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// ------------------------------------------------------------------------------------------------ beside the products

// Copies of matrices whose rows TMA cannot address (unaligned base or stride) in rows that it can, all of a call's in one launch: a warp
// copies 1 KB of a row at a time, words of 4 bytes put together from what the source's alignment allows.
constexpr uint32_t kCopyBytes = 1024;
struct CopyParams {
    struct {
        char *dst;
        const char *src;
        size_t dst_stride, src_stride, first, chunks;     // bytes; number of the first chunk, chunks of a row
        uint32_t bytes;       // of a row
    } m[3];
    uint32_t matrices;
    size_t total;             // chunks
};
template <typename E> __device__ __forceinline__ uint32_t word_of(const char *src, uint32_t left)
{
    uint32_t w = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4; i += sizeof(E))
        if (i < left) w |= uint32_t(*reinterpret_cast<const E *>(src + i)) << 8 * (i % 4);
    return w;
}
__global__ void __launch_bounds__(256) rd_gated_align_kernel(const __grid_constant__ CopyParams p)
{
    pdl_start();
    const uint32_t lane = threadIdx.x & 31;
    for (size_t c = size_t(blockIdx.x) * 8 + (threadIdx.x >> 5); c < p.total; c += size_t(gridDim.x) * 8) {
        const auto &m = p.matrices > 2 && c >= p.m[2].first ? p.m[2] : p.matrices > 1 && c >= p.m[1].first ? p.m[1] : p.m[0];
        const size_t row = (c - m.first) / m.chunks;
        const uint32_t at = uint32_t((c - m.first) % m.chunks) * kCopyBytes + lane * 4;
        const char *src = m.src + row * m.src_stride;
        char *dst = m.dst + row * m.dst_stride;
        const uint32_t odd = uint32_t(reinterpret_cast<uintptr_t>(src)) & 3;
        uint32_t w[kCopyBytes / 128];
#pragma unroll
        for (uint32_t i = 0; i < kCopyBytes / 128; i++) {
            const uint32_t j = at + 128 * i, left = j < m.bytes ? m.bytes - j : 0;
            w[i] = odd & 1 ? word_of<uint8_t>(src + j, left) : odd || left < 4 ? m.bytes & 1 ? word_of<uint8_t>(src + j, left) : word_of<uint16_t>(src + j, left) : word_of<uint32_t>(src + j, left);
        }
        // a word that begins in a row lies in the copy's, which is a multiple of 128 bytes
#pragma unroll
        for (uint32_t i = 0; i < kCopyBytes / 128; i++)
            if (at + 128 * i < m.bytes) *reinterpret_cast<uint32_t *>(dst + at + 128 * i) = w[i];
    }
}

struct SlopeParams {
    const uint16_t *gate, *up, *grad_out;
    size_t gate_stride, up_stride, grad_out_stride;
    uint16_t *both;           // rows of 2 * half values: dgate, zeros up to half, dup, zeros
    size_t n;
    uint32_t width, half, across;
    int act;
    bool bf16;
};

// dgate and dup, V values at a time, as many as the rows' alignment allows.  Where there are enough of them for all threads, a thread has 8
// values of a row in accesses p.across threads apart that are all under way together.  B200, with one access a thread and with these:
// 6550 x 256 x 4978 (pairs of values) 162 and 148 us, 4979 (single ones) 218 and 181, 200 x 1000 x 2730 17.5 and 19.5.
template <int V, int kWords> __global__ void __launch_bounds__(256) rd_gated_slope_kernel(const __grid_constant__ SlopeParams p)
{
    using Word = std::conditional_t<V == 8, uint4, std::conditional_t<V == 2, uint32_t, uint16_t>>;
    constexpr int kPairs = (V + 1) / 2;                  // pairs of values of an access
    union Values {
        Word word;
        uint32_t pair[kPairs];
    };
    pdl_start();
    const uint32_t x = threadIdx.x % p.across, y = threadIdx.x / p.across, down = 256 / p.across, col = (blockIdx.y * p.across * kWords + x) * V, apart = p.across * V;
    for (size_t row = size_t(blockIdx.x) * down + y; row < p.n; row += size_t(gridDim.x) * down) {
        Values g[kWords], u[kWords], d[kWords];
        auto load = [&](Values &v, const uint16_t *matrix, size_t stride, uint32_t j) {
            v.pair[0] = 0;
            if (j < p.width) v.word = *reinterpret_cast<const Word *>(matrix + row * stride + j);
        };
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            load(g[i], p.gate, p.gate_stride, col + i * apart);
            load(u[i], p.up, p.up_stride, col + i * apart);
            load(d[i], p.grad_out, p.grad_out_stride, col + i * apart);
        }
        with_act(p.act, [&](auto ACT) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const uint32_t j = col + i * apart;
                if (j >= p.half) break;
                Values a = {}, b = {};
                if (j < p.width) {
#pragma unroll
                    for (int k = 0; k < kPairs; k++) {
                        const float2 gk = widen2(p.bf16, g[i].pair[k]), uk = widen2(p.bf16, u[i].pair[k]), dk = widen2(p.bf16, d[i].pair[k]);
                        float v0, s0, v1, s1;
                        act_both<decltype(ACT)::value>(gk.x, v0, s0);
                        act_both<decltype(ACT)::value>(gk.y, v1, s1);
                        a.pair[k] = pack2(p.bf16, dk.x * uk.x * s0, dk.y * uk.y * s1);
                        b.pair[k] = pack2(p.bf16, dk.x * v0, dk.y * v1);
                    }
                }
                uint16_t *dst = p.both + row * 2 * p.half + j;
                *reinterpret_cast<Word *>(dst) = a.word;
                *reinterpret_cast<Word *>(dst + p.half) = b.word;
            }
        });
    }
}

// Adds parts of results and rounds: four threads to four columns, each with every fourth part in order, then those in order.
constexpr uint32_t kFinishColumns = 256;
struct FinishParams {
    struct {
        uint16_t *out;
        const float *parts;
        size_t out_stride, step, first;       // step: from one part to the next; number of the first row
        uint32_t splits;
        bool wide;
    } m[3];
    uint32_t matrices, dim, stride;           // stride: of a part's rows, a multiple of 32
    size_t rows;
    bool bf16;
};
__global__ void __launch_bounds__(256) rd_gated_finish_kernel(const __grid_constant__ FinishParams p)
{
    __shared__ float4 sums[3][64];
    pdl_start();
    const uint32_t x = threadIdx.x & 63, y = threadIdx.x >> 6, j = blockIdx.y * kFinishColumns + x * 4;
    for (size_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const auto &m = p.matrices > 2 && r >= p.m[2].first ? p.m[2] : p.matrices > 1 && r >= p.m[1].first ? p.m[1] : p.m[0];
        const size_t row = r - m.first;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (j < p.dim) {
            const float *src = m.parts + row * p.stride + j;
#pragma unroll 8
            for (uint32_t s = y; s < m.splits; s += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(src + s * m.step);
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
        }
        if (y) sums[y - 1][x] = sum;
        __syncthreads();
        if (y == 0 && j < p.dim) {
#pragma unroll
            for (int k = 0; k < 3; k++) {
                const float4 v = sums[k][x];
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
            const uint32_t lo = pack2(p.bf16, sum.x, sum.y), hi = pack2(p.bf16, sum.z, sum.w);
            uint16_t *dst = m.out + row * m.out_stride + j;
            if (m.wide && j + 4 <= p.dim) {
                *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
            } else {
                const uint16_t v[4] = {uint16_t(lo), uint16_t(lo >> 16), uint16_t(hi), uint16_t(hi >> 16)};
#pragma unroll
                for (int k = 0; k < 4; k++)
                    if (j + k < p.dim) dst[k] = v[k];
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------ host

size_t bytes_of(int dtype) { return dtype == RD_E4M3 ? 1 : 2; }

// Bytes between rows that TMA can address: a multiple of 16, as the base.
bool tma_rows(const void *p, size_t stride, size_t esize) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * esize % 16 == 0; }
// An input whose rows are all the same one has no stride that TMA takes, either.
bool tma_input(const void *p, size_t stride, size_t esize) { return tma_rows(p, stride, esize) && stride > 0; }

// Whether pairs of thread blocks compute tiles of twice the rows: as soon as there is more than one tile of 128.
int pair_or_single(size_t n) { return n > kRowsM ? 2 : 1; }
uint32_t rows_in(size_t n) { return uint32_t(n < kRowsM ? round_up(n, 8) : kRowsM); }

struct Layout {
    void *x, *gate_weight, *up_weight;        // aligned copies, null where none is needed
    size_t copy_stride;                       // in elements
    uint16_t *both;
    size_t half;
    float *parts, *parts_w;
    size_t splits, steps_per_split, splits_w, steps_per_split_w, part_stride, part_rows, bytes;
};

// Parts that the sums are cut into, over both widths for dx and over the rows for dWg and dWu.  More parts fill the groups of thread blocks
// more evenly, but each is a matrix of its own that is written and read once more; times in steps of the summed index, of which parts
// have to save a fifth, as groups without work leave the others more power and bandwidth.  B200, without parts and with: 200 x 1000 x 2730
// (6 of dx) 31 / 18 us, 32768 x 512 x 512 (8 of the weights' gradients) 194 / 103, 65536 x 1024 x 1024 (2) 665 / 587, 16384 x 1024 x 4096 (2)
// 573 / 581 and therefore none.
struct Splits {
    size_t x, w;
};
Splits splits_of(const GatedArgs &a, size_t half)
{
    const size_t cg = pair_or_single(a.n), tile_m = kRowsM * cg, groups = kSms / cg, steps_x = 2 * half / kTileK, steps_w = (a.n + kTileK - 1) / kTileK;
    const size_t tiles_n = (a.dim + kTileN - 1) / kTileN, tiles_x = (a.n + tile_m - 1) / tile_m * tiles_n, tiles_w = 2 * ((a.width + tile_m - 1) / tile_m) * tiles_n;
    const double step_bytes = 0.28e-6 * 6.5e12, finish = 9;
    auto steps_of = [](size_t steps, size_t s) { return uint32_t((steps + s - 1) / s); };
    auto most = [&](size_t x, size_t w) {     // steps of the group that gets the most: one with one more unit of dx, or another
        const size_t units_x = tiles_x * x, units_w = tiles_w * w, g = units_x + units_w < groups ? units_x + units_w : groups;
        const uint32_t sx = steps_of(steps_x, x), sw = steps_of(steps_w, w);
        const Deal d(uint32_t(units_x), sx, uint32_t(units_w), sw, uint32_t(g));
        const size_t in_turns = size_t(d.even) * g, others = g - d.more, last = units_w < in_turns ? units_w + g - in_turns : g;   // last: units of the last turn
        const size_t w_more = d.even - (last <= others && last < g), w_others = d.even + (units_w > in_turns ? (units_w - in_turns + others - 1) / others : 0);
        const size_t one_x = sx + kTileOverhead, one_w = sw + kTileOverhead, more = d.more ? (d.dx_each + 1) * one_x + w_more * one_w : 0, other = d.dx_each * one_x + w_others * one_w;
        return double(more > other ? more : other);
    };
    Splits best{1, 1};
    double best_time = 0.8 * most(1, 1);
    for (const size_t x : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64})
        for (const size_t w : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if ((x == 1 && w == 1) || (x > 1 && x * 4 > steps_x) || (w > 1 && w * 4 > steps_w)) continue;
            const double parts = ((x > 1 ? double(x * a.n) : 0) + (w > 1 ? double(w * 2 * a.width) : 0)) * double(a.dim) * 8 / step_bytes + finish;
            if (parts >= best_time) continue;
            const double time = most(x, w) + parts;
            if (time < best_time) best = Splits{x, w}, best_time = time;
        }
    return best;
}

Layout lay_out(const GatedArgs &a, bool gradient, bool want_x)
{
    Layout l{};
    if (a.n == 0) return l;
    Part w(a.workspace);
    const size_t esize = bytes_of(a.dtype);
    l.copy_stride = round_up(a.dim, 128 / esize);
    auto copy = [&](const void *p, size_t stride, size_t rows) -> void * { return tma_input(p, stride, esize) ? nullptr : w.take<char>(rows * l.copy_stride * esize); };
    l.x = copy(a.x, a.x_stride, a.n);
    l.gate_weight = copy(a.gate_weight, a.gate_weight_stride, a.width);
    l.up_weight = copy(a.up_weight, a.up_weight_stride, a.width);
    if (gradient) {
        l.half = round_up(a.width, 64);
        l.both = w.take<uint16_t>(a.n * 2 * l.half);
        // whatever is wanted, so that the bits do not depend on it
        const Splits splits = splits_of(a, l.half);
        auto cut = [](size_t steps, size_t parts, size_t *each, size_t *number) {
            *each = (steps + parts - 1) / parts;
            *number = (steps + *each - 1) / *each;
        };
        cut(2 * l.half / kTileK, splits.x, &l.steps_per_split, &l.splits);
        cut((a.n + kTileK - 1) / kTileK, splits.w, &l.steps_per_split_w, &l.splits_w);
        l.part_stride = round_up(a.dim, 32);
        l.part_rows = round_up(a.width, size_t(kRowsM) * pair_or_single(a.n));
        if (l.splits > 1 && want_x) l.parts = w.take<float>(l.splits * a.n * l.part_stride);
        if (l.splits_w > 1) l.parts_w = w.take<float>(l.splits_w * 2 * l.part_rows * l.part_stride);
    }
    l.bytes = w.at;
    return l;
}

// An operand that TMA can address: the caller's, or its copy, made by this call.
struct Operand {
    const void *p;
    size_t stride;
};
struct Operands {
    Operand x, gate, up;
};
cudaError_t align_all(Operands *o, const GatedArgs &a, const Layout &l)
{
    const size_t esize = bytes_of(a.dtype), chunks = (a.dim * esize + kCopyBytes - 1) / kCopyBytes;
    CopyParams p{};
    auto operand = [&](const void *given, size_t stride, size_t rows, void *copy) {
        if (!copy) return Operand{given, stride};
        p.m[p.matrices++] = {static_cast<char *>(copy), static_cast<const char *>(given), l.copy_stride * esize, stride * esize, p.total, chunks, uint32_t(a.dim * esize)};
        p.total += rows * chunks;
        return Operand{copy, l.copy_stride};
    };
    o->x = operand(a.x, a.x_stride, a.n, l.x);
    o->gate = operand(a.gate_weight, a.gate_weight_stride, a.width, l.gate_weight);
    o->up = operand(a.up_weight, a.up_weight_stride, a.width, l.up_weight);
    if (!p.total) return cudaSuccess;
    const size_t blocks = (p.total + 7) / 8;
    return launch(rd_gated_align_kernel, unsigned(blocks < 8192 ? blocks : 8192), 256, a.stream, p);
}

// A matrix of 8-bit values, read in boxes of 128 values x box_rows rows.
bool encode8(CUtensorMap *map, const void *base, size_t inner, size_t rows, size_t stride, uint32_t box_rows)
{
    const EncodeTiled f = encoder();
    if (!f) return false;
    const cuuint64_t dims[2] = {inner, rows}, strides[1] = {stride};
    const cuuint32_t box[2] = {128, box_rows}, one[2] = {1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool encode_rows(CUtensorMap *map, int dtype, const Operand &o, size_t inner, size_t rows, uint32_t box_rows)
{
    return dtype == RD_E4M3 ? encode8(map, o.p, inner, rows, o.stride, box_rows) : encode(map, dtype == RD_BF16, o.p, inner, rows, o.stride, box_rows);
}

// fp32 accumulators; operand types e4m3 (0), fp16 (0) or bf16 (1); columns and rows of a tile
uint32_t descriptor(int dtype, uint32_t columns, uint32_t rows) { return 1u << 4 | (dtype == RD_BF16 ? 1u << 7 | 1u << 10 : 0u) | columns / 8 << 17 | rows / 16 << 24; }

Out out_of(void *p, size_t stride)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return Out{static_cast<uint16_t *>(p), stride, at % 16 == 0 && stride % 8 == 0 ? 8 : at % 4 == 0 && stride % 2 == 0 ? 2 : 1};
}

// Row tiles that go over the width together: their rows of x (tile x dim) should stay in L2 beside the weights'.
uint32_t row_group(size_t row_bytes, size_t tile_m)
{
    const size_t g = (size_t(32) << 20) / (tile_m * row_bytes);
    return uint32_t(g < 1 ? 1 : g > 64 ? 64 : g);
}

// Columns of a tile (of each projection), a multiple of 8 (pairs: 16, as their products want it): what takes the fewest turns of the groups of thread blocks, by the columns of a
// turn.  Pairs compute narrow tiles at the rate that the left operand comes out of shared memory, as if they had 48 columns.
uint32_t tile_columns(size_t tiles_m, size_t width, size_t groups, bool pairs)
{
    size_t best = 128, best_cost = 0;
    for (size_t w = 128; w >= 16; w -= pairs ? 16 : 8) {
        const size_t turns = (tiles_m * ((width + w - 1) / w) + groups - 1) / groups, cost = turns * ((pairs && w < 48 ? 48 : w) + 8);
        if (w == 128 || cost < best_cost) best = w, best_cost = cost;
    }
    return uint32_t(best);
}

template <bool GRADS, bool F8, int CG, typename P> cudaError_t launch_mma(const P &p, int device, size_t most_units, cudaStream_t stream)
{
    constexpr uint32_t smem = ShapeOf<GRADS, CG>::smem;
    static std::atomic<bool> ready[64];
    if (device >= 64 || !ready[device].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(rd_gated_mma_kernel<GRADS, F8, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
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
    return cudaLaunchKernelEx(&c, rd_gated_mma_kernel<GRADS, F8, CG>, p);
}

}  // namespace

size_t gated_workspace(const GatedArgs &a) { return lay_out(a, false, false).bytes; }

cudaError_t gated_forward(const GatedArgs &a)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const int cg = pair_or_single(a.n);
    const size_t tile_m = size_t(kRowsM) * cg, tiles_m = (a.n + tile_m - 1) / tile_m, esize = bytes_of(a.dtype);
    const Layout l = lay_out(a, false, false);
    Operands o;
    e = align_all(&o, a, l);
    if (e != cudaSuccess) return e;
    GatedParams p{};
    p.n = uint32_t(a.n);
    p.width = uint32_t(a.width);
    p.steps = uint32_t((a.dim * esize + 127) / 128);
    p.tile_w = tile_columns(tiles_m, a.width, kSms / cg, cg == 2);
    p.a_rows = rows_in(a.n);
    p.out = out_of(a.out, a.out_stride);
    p.kept_gate = out_of(a.gate, a.gate_stride);
    p.kept_up = out_of(a.up, a.up_stride);
    // the ring has the room, but for what results change places in
    bool staged = false;
    for (const Out &o : {p.out, p.kept_gate, p.kept_up}) staged |= o.p && o.units != 8;
    const uint32_t room = cg == 2 ? ShapeOf<false, 2>::ring : ShapeOf<false, 1>::ring;
    p.staging = room - kEpilogueWarps * 1024;
    const Ring r = ring_of(staged ? p.staging : room, p.a_rows, 2 * p.tile_w / uint32_t(cg));
    p.stage = r.stage;
    p.stages = r.stages;
    p.group = row_group(a.dim * esize, tile_m);
    p.idesc = descriptor(a.dtype, 2 * p.tile_w, uint32_t(tile_m));
    p.act = a.activation;
    p.bf16 = a.out_dtype == RD_BF16;
    p.x_scale = a.x_scale;
    p.gate_scale = a.gate_scale;
    p.up_scale = a.up_scale;
    if (!encode_rows(&p.a, a.dtype, o.x, a.dim, a.n, p.a_rows) || !encode_rows(&p.gate, a.dtype, o.gate, a.dim, a.width, p.tile_w) ||
        !encode_rows(&p.up, a.dtype, o.up, a.dim, a.width, p.tile_w))
        return cudaErrorInvalidValue;
    const size_t units = tiles_m * ((a.width + p.tile_w - 1) / p.tile_w);
    if (a.dtype == RD_E4M3) return cg == 2 ? launch_mma<false, true, 2>(p, device, units, a.stream) : launch_mma<false, true, 1>(p, device, units, a.stream);
    return cg == 2 ? launch_mma<false, false, 2>(p, device, units, a.stream) : launch_mma<false, false, 1>(p, device, units, a.stream);
}

size_t gated_backward_workspace(const GatedArgs &a, bool want_x) { return lay_out(a, true, want_x).bytes; }

cudaError_t gated_backward(const GatedArgs &a)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const int cg = pair_or_single(a.n);
    const size_t tile_m = size_t(kRowsM) * cg, tiles_m = (a.n + tile_m - 1) / tile_m, tiles_n = (a.dim + kTileN - 1) / kTileN;
    const bool want_x = a.grad_x != nullptr, bf16 = a.dtype == RD_BF16;
    const Layout l = lay_out(a, true, want_x);
    Operands o;
    e = align_all(&o, a, l);
    if (e != cudaSuccess) return e;

    SlopeParams s{};
    s.gate = static_cast<const uint16_t *>(a.gate);
    s.up = static_cast<const uint16_t *>(a.up);
    s.grad_out = static_cast<const uint16_t *>(a.grad_out);
    s.gate_stride = a.gate_stride;
    s.up_stride = a.up_stride;
    s.grad_out_stride = a.grad_out_stride;
    s.both = l.both;
    s.n = a.n;
    s.width = uint32_t(a.width);
    s.half = uint32_t(l.half);
    s.act = a.activation;
    s.bf16 = bf16;
    // values that an access takes
    int v = a.width % 8 == 0 ? 8 : a.width % 2 == 0 ? 2 : 1;
    for (const auto &m : {Operand{a.gate, a.gate_stride}, Operand{a.up, a.up_stride}, Operand{a.grad_out, a.grad_out_stride}})
        while (v > 1 && (reinterpret_cast<uintptr_t>(m.p) % (2 * v) != 0 || m.stride % v != 0)) v = v == 8 ? 2 : 1;
    const bool many = a.n * s.half >= kSms * 1024 * 8;   // half of the threads that there can be, with 8 values each
    const uint32_t units = s.half / (many ? 8 : v);      // threads to a row
    s.across = 256;
    while (s.across > 8 && s.across >= 2 * units) s.across /= 2;
    const size_t down = 256 / s.across, tall = (a.n + down - 1) / down;
    const dim3 grid(unsigned(tall < 65536 ? tall : 65536), (units + s.across - 1) / s.across);
    void (*const slope)(SlopeParams) = v == 8 ? rd_gated_slope_kernel<8, 1> : v == 2 ? many ? rd_gated_slope_kernel<2, 4> : rd_gated_slope_kernel<2, 1>
                                                                              : many ? rd_gated_slope_kernel<1, 8> : rd_gated_slope_kernel<1, 1>;
    e = launch(slope, grid, 256, a.stream, s);
    if (e != cudaSuccess) return e;

    GradParams p{};
    p.n = uint32_t(a.n);
    p.dim = uint32_t(a.dim);
    p.width = uint32_t(a.width);
    p.half = uint32_t(l.half);
    p.splits = uint32_t(l.splits);
    p.steps_per_split = uint32_t(l.steps_per_split);
    p.splits_w = uint32_t(l.splits_w);
    p.steps_per_split_w = uint32_t(l.steps_per_split_w);
    p.part_rows = uint32_t(l.part_rows);
    p.a_rows = rows_in(a.n);
    p.idesc = descriptor(a.dtype, kTileN, uint32_t(tile_m));
    p.weights = (a.grad_gate_weight ? 1u : 0u) | (a.grad_up_weight ? 2u : 0u);
    p.want_dx = want_x;
    p.bf16 = bf16;
    p.dx = static_cast<uint16_t *>(a.grad_x);
    p.dgate = static_cast<uint16_t *>(a.grad_gate_weight);
    p.dup = static_cast<uint16_t *>(a.grad_up_weight);
    p.dx_stride = a.grad_x_stride;
    p.dgate_stride = a.grad_gate_weight_stride;
    p.dup_stride = a.grad_up_weight_stride;
    p.dx_tma = want_x && tma_rows(a.grad_x, a.grad_x_stride, 2);
    p.gate_tma = a.grad_gate_weight && tma_rows(a.grad_gate_weight, a.grad_gate_weight_stride, 2);
    p.up_tma = a.grad_up_weight && tma_rows(a.grad_up_weight, a.grad_up_weight_stride, 2);
    if (!encode(&p.a_k, bf16, l.both, 2 * l.half, a.n, 2 * l.half, p.a_rows) || !encode(&p.a_mn, bf16, l.both, 2 * l.half, a.n, 2 * l.half, 64) ||
        !encode(&p.gate_mn, bf16, o.gate.p, a.dim, a.width, o.gate.stride, 64) || !encode(&p.up_mn, bf16, o.up.p, a.dim, a.width, o.up.stride, 64) ||
        !encode(&p.x_mn, bf16, o.x.p, a.dim, a.n, o.x.stride, 64) || (p.dx_tma && !encode(&p.dx_out, bf16, a.grad_x, a.dim, a.n, a.grad_x_stride, 32)) ||
        (p.gate_tma && !encode(&p.gate_out, bf16, a.grad_gate_weight, a.dim, a.width, a.grad_gate_weight_stride, 32)) ||
        (p.up_tma && !encode(&p.up_out, bf16, a.grad_up_weight, a.dim, a.width, a.grad_up_weight_stride, 32)) ||
        (l.parts && !encode_dh(&p.dx_parts, l.parts, l.part_stride, a.n, l.splits)) ||
        (l.parts_w && !encode_dh(&p.dw_parts, l.parts_w, l.part_stride, 2 * l.part_rows, l.splits_w)))
        return cudaErrorInvalidValue;
    const size_t work = (want_x ? tiles_m * tiles_n * l.splits : 0) + __builtin_popcount(p.weights) * ((a.width + tile_m - 1) / tile_m) * tiles_n * l.splits_w;
    e = cg == 2 ? launch_mma<true, false, 2>(p, device, work, a.stream) : launch_mma<true, false, 1>(p, device, work, a.stream);
    if (e != cudaSuccess) return e;
    FinishParams f{};
    auto add = [&](void *out, size_t stride, const float *parts, size_t rows, size_t part_rows, size_t splits) {
        f.m[f.matrices++] = {static_cast<uint16_t *>(out), parts, stride, part_rows * l.part_stride, f.rows, uint32_t(splits), reinterpret_cast<uintptr_t>(out) % 8 == 0 && stride % 4 == 0};
        f.rows += rows;
    };
    if (want_x && l.parts) add(a.grad_x, a.grad_x_stride, l.parts, a.n, a.n, l.splits);
    if (a.grad_gate_weight && l.parts_w) add(a.grad_gate_weight, a.grad_gate_weight_stride, l.parts_w, a.width, 2 * l.part_rows, l.splits_w);
    if (a.grad_up_weight && l.parts_w) add(a.grad_up_weight, a.grad_up_weight_stride, l.parts_w + l.part_rows * l.part_stride, a.width, 2 * l.part_rows, l.splits_w);
    if (!f.rows) return e;
    f.dim = uint32_t(a.dim);
    f.stride = uint32_t(l.part_stride);
    f.bf16 = bf16;
    return launch(rd_gated_finish_kernel, dim3(unsigned(f.rows < 65536 ? f.rows : 65536), unsigned((a.dim + kFinishColumns - 1) / kFinishColumns)), 256, a.stream, f);
}

cudaError_t block_status(int *status)
{
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return e;
    int of_norm = 0;
    e = norm_status(&of_norm);
    if (e != cudaSuccess) return e;
    e = cudaMemcpyFromSymbol(status, g_wait_status, sizeof(int));
    if (e != cudaSuccess) return e;
    const int zero = 0;
    if (*status) e = cudaMemcpyToSymbol(g_wait_status, &zero, sizeof(int));
    *status |= of_norm;
    return e;
}

}  // namespace rd
