// sm_100a kernels of the root-mean-square norm with the residual's addition and dropout, of its gradient, and of dropout alone.
//
//   s = residual + keep x,   r = 1 / sqrt(mean s^2 + eps),   out = s r w          (8 bits: scale = max |out| / 448, out / scale)
//   xhat = s r,  g = grad_out w:   grad = r (g - xhat mean(g xhat)) + grad_sum,   grad_x = keep grad,   grad_w = sum over rows of grad_out xhat
//
// keep is 65536 / (65536 - border) where a value's 16 random bits reach the border, else 0.  The bits are those of Philox 4x32 with
// 10 rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), whose counter is the value's place:
// (column / 8, row, offset), key: the seed.  So a mask is never stored; whoever knows the place knows the bits.
//
// A row is held in registers from its loads to its stores: by a warp up to 1024 values, by a thread block up to 8192, above by a
// cluster of up to eight of them, whose partial sums meet in each other's shared memory.  Everything is read and written once.
// What bounds it: the memory; a single row, the latency of a launch, a load, a reduction and a store.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "rd.h"
#include "rd_block.h"
#include "rd_launch.h"

namespace rd {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kWarpDim = 1024;       // rows up to here are a warp's
constexpr uint32_t kBlockDim = 8192;      // a thread block's part of a row at most: 32 values a thread
constexpr size_t kSms = 148;

struct F32 {
    static constexpr int words = 8;       // of 8 values
};
struct B16 {
    static constexpr int words = 4;
};
struct H16 {
    static constexpr int words = 4;
};

// V values (8, or 1 where rows are not made of 16-byte words) as they lie in memory.
template <class T, int V> struct Pack {
    uint32_t w[V == 8 ? T::words : 1];
    __device__ __forceinline__ void load(const void *base, size_t at)
    {
        if constexpr (V == 8) {
            const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + at * (T::words / 2));
#pragma unroll
            for (int i = 0; i < T::words / 4; i++) {
                const uint4 v = p[i];
                w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
            }
        } else if constexpr (T::words == 8) {
            w[0] = static_cast<const uint32_t *>(base)[at];
        } else {
            w[0] = static_cast<const uint16_t *>(base)[at];
        }
    }
    __device__ __forceinline__ void store(void *base, size_t at) const
    {
        if constexpr (V == 8) {
            uint4 *p = reinterpret_cast<uint4 *>(static_cast<char *>(base) + at * (T::words / 2));
#pragma unroll
            for (int i = 0; i < T::words / 4; i++) p[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else if constexpr (T::words == 8) {
            static_cast<uint32_t *>(base)[at] = w[0];
        } else {
            static_cast<uint16_t *>(base)[at] = uint16_t(w[0]);
        }
    }
    __device__ __forceinline__ void get(float (&f)[V]) const
    {
        if constexpr (T::words == 8) {
#pragma unroll
            for (int i = 0; i < V; i++) f[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < (V + 1) / 2; i++) {
                float2 v;
                if constexpr (std::is_same_v<T, B16>) v = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
                else v = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                f[2 * i] = v.x;
                if (V > 1) f[2 * i + 1 < V ? 2 * i + 1 : 0] = v.y;
            }
        }
    }
    __device__ __forceinline__ void set(const float (&f)[V])
    {
        if constexpr (T::words == 8) {
#pragma unroll
            for (int i = 0; i < V; i++) w[i] = __float_as_uint(f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < (V + 1) / 2; i++) {
                const float lo = f[2 * i], hi = V > 1 ? f[2 * i + 1 < V ? 2 * i + 1 : 0] : 0.0f;
                if constexpr (std::is_same_v<T, B16>) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(hi), "f"(lo));
                else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(hi), "f"(lo));
            }
        }
    }
};

// The weight, in the rows' type or in 32 bits.
template <class T, int V> __device__ __forceinline__ void get_weight(const void *weight, bool wide, size_t at, float (&w)[V])
{
    if (wide) {
        Pack<F32, V> p;
        p.load(weight, at);
        p.get(w);
    } else {
        Pack<T, V> p;
        p.load(weight, at);
        p.get(w);
    }
}

struct Drop {
    uint32_t border;
    float keep;
    uint32_t key0, key1, offset0, offset1, first;
};

// The 128 random bits of 8 columns of a row.
__device__ __forceinline__ uint4 random_bits(const Drop &d, uint32_t unit, uint32_t row)
{
    uint32_t a = unit, b = row, c = d.offset0, e = d.offset1, k0 = d.key0, k1 = d.key1;
#pragma unroll
    for (int i = 0; i < 10; i++) {
        const uint32_t ha = __umulhi(0xD2511F53u, a), la = 0xD2511F53u * a, hc = __umulhi(0xCD9E8D57u, c), lc = 0xCD9E8D57u * c;
        a = hc ^ b ^ k0;
        b = lc;
        c = ha ^ e ^ k1;
        e = la;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(a, b, c, e);
}
__device__ __forceinline__ float kept(const Drop &d, uint32_t bits, float x) { return bits >= d.border ? x * d.keep : 0.0f; }

// Dropout of the V values of a row from column `column` on.
template <int V> __device__ __forceinline__ void drop_values(const Drop &d, uint32_t column, size_t row, float (&x)[V])
{
    const uint4 r = random_bits(d, column / 8, uint32_t(row) + d.first);
    if constexpr (V == 8) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = kept(d, i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu, x[i]);
    } else {
        const uint32_t at = column % 8, w = at < 4 ? (at < 2 ? r.x : r.y) : (at < 6 ? r.z : r.w);
        x[0] = kept(d, at & 1 ? w >> 16 : w & 0xffffu, x[0]);
    }
}

// ------------------------------------------------------------------------------------------------ sums over a row

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

struct Meeting {
    float2 of_warp[2][kWarps];
    float2 of_block[2][8];
};

// (sum, maximum) over the threads of a row: a warp, or `blocks` thread blocks of a cluster.  Two sets of places take turns: whoever
// writes to one has seen every thread arrive after its last reading.
template <bool WARP> __device__ __forceinline__ float2 join_row(float2 v, Meeting &m, uint32_t turn, uint32_t blocks, uint32_t rank)
{
#pragma unroll
    for (int d = 16; d; d /= 2) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
        v.y = fmaxf(v.y, __shfl_xor_sync(0xffffffffu, v.y, d));
    }
    if (WARP) return v;
    const uint32_t set = turn & 1;
    if ((threadIdx.x & 31) == 0) m.of_warp[set][threadIdx.x >> 5] = v;
    __syncthreads();
    v = m.of_warp[set][0];
#pragma unroll
    for (int k = 1; k < kWarps; k++) {
        const float2 o = m.of_warp[set][k];
        v = make_float2(v.x + o.x, fmaxf(v.y, o.y));
    }
    if (blocks == 1) return v;
    if (threadIdx.x < blocks) {
        const uint32_t here = uint32_t(__cvta_generic_to_shared(&m.of_block[set][rank]));
        uint32_t there;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(threadIdx.x));
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.x), "f"(v.y) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    v = m.of_block[set][0];
    for (uint32_t k = 1; k < blocks; k++) {
        const float2 o = m.of_block[set][k];
        v = make_float2(v.x + o.x, fmaxf(v.y, o.y));
    }
    return v;
}

// Which rows and which units of V values of them a thread has.
template <int V, bool WARP> struct Place {
    size_t row, rows;         // first row, and how many rows further the next is
    uint32_t unit, end, rank;
    __device__ __forceinline__ Place(uint32_t units, uint32_t per_block, uint32_t blocks)
    {
        if (WARP) {
            row = size_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
            rows = size_t(gridDim.x) * kWarps;
            unit = threadIdx.x & 31;
            end = units;
            rank = 0;
        } else {
            rank = blocks > 1 ? cluster_rank() : 0;
            row = blockIdx.x / blocks;
            rows = gridDim.x / blocks;
            unit = rank * per_block + threadIdx.x;
            end = min(units, (rank + 1) * per_block);
        }
    }
    static constexpr uint32_t step = WARP ? 32 : kThreads;
};

struct NormParams {
    const void *x, *residual, *weight;
    void *out, *sum;
    float *out_scale, *rstd;
    size_t x_stride, residual_stride, out_stride, sum_stride, n;
    uint32_t units, per_block, blocks;
    float eps, inv_dim;
    Drop drop;
    bool wide_weight, out8;
};

// T: x and out, R: residual and sum.  A thread holds NV units of V values of a row.
template <class T, class R, int V, int NV, bool WARP> __global__ void __launch_bounds__(kThreads) rd_norm_kernel(const __grid_constant__ NormParams p)
{
    __shared__ Meeting meeting;
    pdl_start();
    const Place<V, WARP> at(p.units, p.per_block, p.blocks);
    uint32_t turn = 0;
    for (size_t row = at.row; row < p.n; row += at.rows, turn++) {
        Pack<T, V> x[NV];
        Pack<R, V> res[NV];
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.unit + k * at.step < at.end) {
                x[k].load(p.x, row * p.x_stride + size_t(at.unit + k * at.step) * V);
                if (p.residual) res[k].load(p.residual, row * p.residual_stride + size_t(at.unit + k * at.step) * V);
            }
        float s[NV][V];
        float2 stat = make_float2(0.0f, 0.0f);        // sum of squares, largest |s w|
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.unit + k * at.step < at.end) {
                const uint32_t column = (at.unit + k * at.step) * V;
                x[k].get(s[k]);
                if (p.drop.border) drop_values<V>(p.drop, column, row, s[k]);
                if (p.residual) {
                    float r[V];
                    res[k].get(r);
#pragma unroll
                    for (int i = 0; i < V; i++) s[k][i] += r[i];
                }
                if (p.sum) {
                    Pack<R, V> o;
                    o.set(s[k]);
                    o.store(p.sum, row * p.sum_stride + column);
                }
                float w[V];
                get_weight<T, V>(p.weight, p.wide_weight, column, w);
#pragma unroll
                for (int i = 0; i < V; i++) {
                    stat.x = fmaf(s[k][i], s[k][i], stat.x);
                    s[k][i] *= w[i];
                    stat.y = fmaxf(stat.y, fabsf(s[k][i]));
                }
            }
        stat = join_row<WARP>(stat, meeting, turn, p.blocks, at.rank);
        const float rstd = rsqrtf(fmaf(stat.x, p.inv_dim, p.eps));
        float factor = rstd;
        if (p.out8) {
            // the row's largest value becomes 448; very small ones are taken near 1 first, so that no quotient overflows
            const float lift = stat.y < 0x1p-60f ? 0x1p64f : 1.0f;
            factor = stat.y > 0.0f ? 448.0f / (stat.y * lift) : 0.0f;
            if (lift != 1.0f) {
#pragma unroll
                for (int k = 0; k < NV; k++)
#pragma unroll
                    for (int i = 0; i < V; i++) s[k][i] *= lift;
            }
        }
        if (at.unit == (WARP ? 0 : at.rank * p.per_block) && at.rank == 0) {
            if (p.rstd) p.rstd[row] = rstd;
            if (p.out8) p.out_scale[row] = stat.y * rstd / 448.0f;
        }
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.unit + k * at.step < at.end) {
                const size_t to = row * p.out_stride + size_t(at.unit + k * at.step) * V;
#pragma unroll
                for (int i = 0; i < V; i++) s[k][i] *= factor;
                if (p.out8) {
                    if constexpr (V == 8) {
                        uint16_t q[4];
#pragma unroll
                        for (int i = 0; i < 4; i++) q[i] = __nv_cvt_float2_to_fp8x2(make_float2(s[k][2 * i], s[k][2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
                        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.out) + to) = make_uint2(q[0] | uint32_t(q[1]) << 16, q[2] | uint32_t(q[3]) << 16);
                    } else {
                        static_cast<uint8_t *>(p.out)[to] = __nv_cvt_float_to_fp8(s[k][0], __NV_SATFINITE, __NV_E4M3);
                    }
                } else {
                    Pack<T, V> o;
                    o.set(s[k]);
                    o.store(p.out, to);
                }
            }
    }
}

// ------------------------------------------------------------------------------------------------ gradient

struct NormGradParams {
    const void *grad_out, *sum, *weight, *grad_sum;
    const float *rstd;
    void *grad_x, *grad_residual;
    float *part;              // [groups][dim]: every group's part of grad_weight; null where it is not wanted
    size_t grad_out_stride, sum_stride, grad_sum_stride, grad_x_stride, grad_residual_stride, n;
    uint32_t units, per_block, blocks, dim;
    float inv_dim;
    Drop drop;
    bool wide_weight, want_rows;
};

// Persistent groups of threads that take rows in turn; a thread's columns stay the same, so that grad_weight adds up in its registers.
template <class T, class R, int V, int NV, bool WARP> __global__ void __launch_bounds__(kThreads) rd_norm_grad_kernel(const __grid_constant__ NormGradParams p)
{
    __shared__ Meeting meeting;
    pdl_start();
    const Place<V, WARP> at(p.units, p.per_block, p.blocks);
    float acc[NV][V] = {};
    uint32_t turn = 0;
    for (size_t row = at.row; row < p.n; row += at.rows, turn++) {
        Pack<T, V> up[NV];
        Pack<R, V> sum[NV], more[NV];
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.unit + k * at.step < at.end) {
                const size_t column = size_t(at.unit + k * at.step) * V;
                up[k].load(p.grad_out, row * p.grad_out_stride + column);
                sum[k].load(p.sum, row * p.sum_stride + column);
                if (p.grad_sum && p.want_rows) more[k].load(p.grad_sum, row * p.grad_sum_stride + column);
            }
        const float rstd = p.rstd[row];
        float2 stat = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.unit + k * at.step < at.end) {
                float u[V], s[V], w[V];
                up[k].get(u);
                sum[k].get(s);
                get_weight<T, V>(p.weight, p.wide_weight, size_t(at.unit + k * at.step) * V, w);
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float y = u[i] * (s[i] * rstd);
                    acc[k][i] += y;
                    stat.x = fmaf(y, w[i], stat.x);
                }
            }
        if (!p.want_rows) continue;
        const float mean = join_row<WARP>(stat, meeting, turn, p.blocks, at.rank).x * p.inv_dim;
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.unit + k * at.step < at.end) {
                const uint32_t column = (at.unit + k * at.step) * V;
                float u[V], s[V], w[V];
                up[k].get(u);
                sum[k].get(s);
                get_weight<T, V>(p.weight, p.wide_weight, column, w);
#pragma unroll
                for (int i = 0; i < V; i++) u[i] = rstd * fmaf(-mean, s[i] * rstd, u[i] * w[i]);
                if (p.grad_sum) {
                    float m[V];
                    more[k].get(m);
#pragma unroll
                    for (int i = 0; i < V; i++) u[i] += m[i];
                }
                if (p.grad_residual) {
                    Pack<R, V> o;
                    o.set(u);
                    o.store(p.grad_residual, row * p.grad_residual_stride + column);
                }
                if (p.grad_x) {
                    if (p.drop.border) drop_values<V>(p.drop, column, row, u);
                    Pack<T, V> o;
                    o.set(u);
                    o.store(p.grad_x, row * p.grad_x_stride + column);
                }
            }
    }
    if (!p.part) return;
    if constexpr (WARP) {
        // the block's warps, one after the other in shared memory, in order
        __shared__ float of_warp[kWarps][kWarpDim];
        const uint32_t warp = threadIdx.x >> 5;
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.unit + k * at.step < at.end)
#pragma unroll
                for (int i = 0; i < V; i++) of_warp[warp][(at.unit + k * at.step) * V + i] = acc[k][i];
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < p.dim; j += kThreads) {
            float v = of_warp[0][j];
#pragma unroll
            for (int k = 1; k < kWarps; k++) v += of_warp[k][j];
            p.part[size_t(blockIdx.x) * p.dim + j] = v;
        }
    } else {
        float *dst = p.part + size_t(blockIdx.x / p.blocks) * p.dim;
#pragma unroll
        for (int k = 0; k < NV; k++)
            if (at.unit + k * at.step < at.end) {
                Pack<F32, V> o;
                o.set(acc[k]);
                o.store(dst, size_t(at.unit + k * at.step) * V);
            }
    }
}

// Adds up the groups' parts: 32 columns a block, each by 32 threads that take every 32nd part, then those in order.
constexpr int kJoinThreads = 1024;
template <class W> __global__ void __launch_bounds__(kJoinThreads) rd_norm_weight_kernel(void *grad_weight, const float *part, uint32_t parts, uint32_t dim)
{
    __shared__ float of_lane[32][33];
    pdl_start();
    const uint32_t column = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
    float v = 0.0f;
    if (column < dim)
#pragma unroll 8
        for (uint32_t k = lane; k < parts; k += 32) v += part[size_t(k) * dim + column];
    of_lane[threadIdx.x & 31][lane] = v;
    __syncthreads();
    // a warp per column
    v = of_lane[lane][threadIdx.x & 31];
#pragma unroll
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0 && blockIdx.x * 32 + lane < dim) {
        Pack<W, 1> o;
        const float f[1] = {v};
        o.set(f);
        o.store(grad_weight, blockIdx.x * 32 + lane);
    }
}

// ------------------------------------------------------------------------------------------------ dropout alone

struct DropoutParams {
    const void *x;
    void *out;
    size_t x_stride, out_stride, n;
    uint32_t units, across;   // threads that a row's units are dealt out to; the block's others have rows of their own
    Drop drop;
};

template <class T, int V> __global__ void __launch_bounds__(kThreads) rd_dropout_kernel(const __grid_constant__ DropoutParams p)
{
    pdl_start();
    const uint32_t x = threadIdx.x % p.across, y = threadIdx.x / p.across, down = kThreads / p.across;
    const uint32_t unit0 = blockIdx.y * p.across * 4 + x;
    for (size_t row = size_t(blockIdx.x) * down + y; row < p.n; row += size_t(gridDim.x) * down) {
        Pack<T, V> v[4];
#pragma unroll
        for (int k = 0; k < 4; k++)
            if (unit0 + k * p.across < p.units) v[k].load(p.x, row * p.x_stride + size_t(unit0 + k * p.across) * V);
#pragma unroll
        for (int k = 0; k < 4; k++)
            if (unit0 + k * p.across < p.units) {
                const uint32_t column = (unit0 + k * p.across) * V;
                float f[V];
                v[k].get(f);
                drop_values<V>(p.drop, column, row, f);
                v[k].set(f);
                v[k].store(p.out, row * p.out_stride + column);
            }
    }
}

// ------------------------------------------------------------------------------------------------ host

Drop drop_of(const DropArgs &d)
{
    return Drop{d.border, d.keep, uint32_t(d.seed), uint32_t(d.seed >> 32), uint32_t(d.offset), uint32_t(d.offset >> 32), d.first};
}

size_t size_of(int dtype) { return dtype == RD_FP32 ? 4 : dtype == RD_E4M3 ? 1 : 2; }

// Whether a matrix's rows are made of units of 8 values that one or two 16-byte accesses (8 bits: one of 8 bytes) take.
bool in_units(const void *p, size_t stride, int dtype)
{
    const size_t to = dtype == RD_E4M3 ? 8 : 16;
    return !p || (reinterpret_cast<uintptr_t>(p) % to == 0 && stride * size_of(dtype) % to == 0);
}

// How a row is dealt out.
struct Deal {
    uint32_t units, per_block, blocks;
    int nv;                   // units a thread
    bool warp;
};
Deal deal(size_t dim, int v)
{
    Deal d{};
    d.units = uint32_t((dim + v - 1) / v);
    d.warp = dim <= kWarpDim;
    d.blocks = 1;
    while (!d.warp && (d.units + d.blocks - 1) / d.blocks * v > kBlockDim) d.blocks *= 2;
    d.per_block = (d.units + d.blocks - 1) / d.blocks;
    const uint32_t threads = d.warp ? 32 : kThreads, most = (d.per_block + threads - 1) / threads;
    d.nv = v == 1 ? 32 : most <= 1 ? 1 : most <= 2 ? 2 : 4;
    return d;
}

template <typename P> cudaError_t launch_rows(void (*kernel)(P), const P &p, size_t groups, uint32_t blocks, cudaStream_t stream)
{
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(unsigned(groups * blocks));
    c.blockDim = dim3(kThreads);
    c.stream = stream;
    cudaLaunchAttribute attrs[2] = {pdl_attribute()};
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = blocks;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    c.attrs = attrs;
    c.numAttrs = blocks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&c, kernel, p);
}

// Calls f with the kernel's template arguments: how the row lies, then the types.
template <class F> cudaError_t with_shape(int v, int nv, bool warp, F &&f)
{
    using std::integral_constant;
    auto with = [&](auto V, auto NV) { return warp ? f(V, NV, integral_constant<bool, true>()) : f(V, NV, integral_constant<bool, false>()); };
    if (v == 1) return with(integral_constant<int, 1>(), integral_constant<int, 32>());
    if (nv == 1) return with(integral_constant<int, 8>(), integral_constant<int, 1>());
    if (nv == 2) return with(integral_constant<int, 8>(), integral_constant<int, 2>());
    return with(integral_constant<int, 8>(), integral_constant<int, 4>());
}
template <class F> cudaError_t with_types(int dtype, int sum_dtype, F &&f)
{
    if (dtype == RD_FP32) return f(F32(), F32());
    if (dtype == RD_BF16) return sum_dtype == RD_FP32 ? f(B16(), F32()) : f(B16(), B16());
    return sum_dtype == RD_FP32 ? f(H16(), F32()) : f(H16(), H16());
}

// Groups of threads (a warp or a cluster has a row at a time) that the gradient keeps busy, and whose parts of grad_weight there are.
size_t grad_blocks(size_t n, const Deal &d)
{
    const size_t rows = d.warp ? kWarps : 1, wanted = (n + rows - 1) / rows, most = kSms * 3 / d.blocks;
    return wanted < most ? wanted : most;
}

}  // namespace

cudaError_t norm_forward(const NormArgs &a)
{
    const int v = a.dim % 8 == 0 && in_units(a.x, a.x_stride, a.dtype) && in_units(a.residual, a.residual_stride, a.sum_dtype) && in_units(a.weight, 0, a.weight_dtype) &&
                          in_units(a.out, a.out_stride, a.out_dtype) && in_units(a.sum, a.sum_stride, a.sum_dtype)
                      ? 8
                      : 1;
    const Deal d = deal(a.dim, v);
    NormParams p{};
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
    p.units = d.units;
    p.per_block = d.per_block;
    p.blocks = d.blocks;
    p.eps = a.eps;
    p.inv_dim = 1.0f / float(a.dim);
    p.drop = drop_of(a.drop);
    p.wide_weight = a.weight_dtype == RD_FP32;
    p.out8 = a.out_dtype == RD_E4M3;
    const size_t wanted = d.warp ? (a.n + kWarps - 1) / kWarps : a.n, most = kSms * 16 / d.blocks, groups = wanted < most ? wanted : most;
    return with_shape(v, d.nv, d.warp, [&](auto V, auto NV, auto WARP) {
        return with_types(a.dtype, a.sum_dtype, [&](auto T, auto R) { return launch_rows(rd_norm_kernel<decltype(T), decltype(R), V(), NV(), WARP()>, p, groups, d.blocks, a.stream); });
    });
}

size_t norm_backward_workspace(size_t n, size_t dim)
{
    // rows that are not made of 16-byte words are dealt out to as many groups
    const size_t parts = grad_blocks(n, deal(dim, 1)), more = grad_blocks(n, deal((dim + 7) / 8 * 8, 8));
    return (parts > more ? parts : more) * dim * sizeof(float);
}

cudaError_t norm_backward(const NormGradArgs &a)
{
    const int v = a.dim % 8 == 0 && in_units(a.grad_out, a.grad_out_stride, a.dtype) && in_units(a.sum, a.sum_stride, a.sum_dtype) && in_units(a.weight, 0, a.weight_dtype) &&
                          in_units(a.grad_sum, a.grad_sum_stride, a.sum_dtype) && in_units(a.grad_x, a.grad_x_stride, a.dtype) &&
                          in_units(a.grad_residual, a.grad_residual_stride, a.sum_dtype)
                      ? 8
                      : 1;
    const Deal d = deal(a.dim, v);
    const size_t groups = grad_blocks(a.n, d);
    NormGradParams p{};
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
    p.units = d.units;
    p.per_block = d.per_block;
    p.blocks = d.blocks;
    p.dim = uint32_t(a.dim);
    p.inv_dim = 1.0f / float(a.dim);
    p.drop = drop_of(a.drop);
    p.wide_weight = a.weight_dtype == RD_FP32;
    p.want_rows = a.grad_x || a.grad_residual;
    cudaError_t e = cudaSuccess;
    if (groups)
        e = with_shape(v, d.nv, d.warp, [&](auto V, auto NV, auto WARP) {
            return with_types(a.dtype, a.sum_dtype,
                              [&](auto T, auto R) { return launch_rows(rd_norm_grad_kernel<decltype(T), decltype(R), V(), NV(), WARP()>, p, groups, d.blocks, a.stream); });
        });
    if (e != cudaSuccess || !a.grad_weight) return e;
    auto *join = a.weight_dtype == RD_FP32 ? rd_norm_weight_kernel<F32> : a.weight_dtype == RD_BF16 ? rd_norm_weight_kernel<B16> : rd_norm_weight_kernel<H16>;
    return launch(join, unsigned((a.dim + 31) / 32), kJoinThreads, a.stream, a.grad_weight, static_cast<const float *>(a.workspace), uint32_t(groups), uint32_t(a.dim));
}

cudaError_t dropout(const DropoutArgs &a)
{
    const int v = a.dim % 8 == 0 && in_units(a.x, a.x_stride, a.dtype) && in_units(a.out, a.out_stride, a.dtype) ? 8 : 1;
    DropoutParams p{};
    p.x = a.x;
    p.out = a.out;
    p.x_stride = a.x_stride;
    p.out_stride = a.out_stride;
    p.n = a.n;
    p.units = uint32_t((a.dim + v - 1) / v);
    p.across = kThreads;
    while (p.across > 8 && p.across * 2 > p.units) p.across /= 2;      // so that most threads have two units or more
    p.drop = drop_of(a.drop);
    const uint32_t down = kThreads / p.across;
    const size_t tall = (a.n + down - 1) / down;
    const dim3 grid(unsigned(tall < 65536 ? tall : 65536), (p.units + 4 * p.across - 1) / (4 * p.across));
    auto run = [&](auto T) {
        using Type = decltype(T);
        return v == 8 ? launch(rd_dropout_kernel<Type, 8>, grid, kThreads, a.stream, p) : launch(rd_dropout_kernel<Type, 1>, grid, kThreads, a.stream, p);
    };
    return a.dtype == RD_FP32 ? run(F32()) : a.dtype == RD_BF16 ? run(B16()) : run(H16());
}

}  // namespace rd
