// Rows of the norm and of its gradient: how they are dealt out, brought in, summed and dropped from.
#ifndef RD_NORM_ROWS_H_
#define RD_NORM_ROWS_H_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>
#include <type_traits>

#include "rd.h"
#include "rd_block.h"
#include "rd_launch.h"
#include "rd_norm_shape.h"
#include "rd_ptx.h"

namespace rd {

namespace {

__device__ int g_wait_status;             // a wait that was given up

__device__ __forceinline__ const void *at_byte(const void *p, size_t at) { return static_cast<const char *>(p) + at; }
__device__ __forceinline__ void *at_byte(void *p, size_t at) { return static_cast<char *>(p) + at; }

// Two fp32 values in a register pair, and the operations that take both at once (each rounded like the single one).
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 both(Pair v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ Pair add2(Pair x, Pair y)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair x, Pair y)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair x, Pair y, Pair z)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}

// Columns are dealt out in units of 8, a thread's value i of unit u being
//   column 8 u + i, where rows are made of whole units and begin on 16-byte boundaries (fp32: 32): one access of 16 or 32 bytes;
//   otherwise (SPREAD) column 32 i + u mod 32 of the 256 columns that a warp's 32 units are: accesses by element, side by side.
template <bool SPREAD> __device__ __forceinline__ uint32_t column_of(uint32_t unit, int i) { return SPREAD ? (unit & ~31u) * 8 + (unit & 31u) + 32 * i : unit * 8 + i; }

// A thread's 8 values of a unit, as they lie in memory.
template <class T, bool SPREAD> struct Unit {
    static constexpr uint32_t bytes = 4 * T::words;
    uint32_t w[T::words];
    // `row`: where the row begins; zeros where there is nothing to read.  SHARED: in shared memory
    template <bool SHARED = false> __device__ __forceinline__ void load(const void *row, uint32_t unit, uint32_t dim, bool there)
    {
#pragma unroll
        for (int i = 0; i < T::words; i++) w[i] = 0;
        if (!there) return;
        if constexpr (!SPREAD && !SHARED && T::words == 8) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                         : "l"(static_cast<const char *>(row) + unit * bytes));
        } else if constexpr (!SPREAD) {
            const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const char *>(row) + unit * bytes);
#pragma unroll
            for (int i = 0; i < T::words / 4; i++) {
                const uint4 v = p[i];
                w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
            }
        } else {
            using E = std::conditional_t<T::words == 8, uint32_t, uint16_t>;
            const uint32_t first = column_of<true>(unit, 0);
            const E *p = static_cast<const E *>(row) + first;
            E v[8];
            if ((unit & ~31u) * 8 + 256 <= dim) {          // all of the warp's columns
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] = p[32 * i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] = first + 32 * i < dim ? p[32 * i] : E(0);
            }
#pragma unroll
            for (int i = 0; i < T::words; i++) w[i] = T::words == 8 ? v[i] : v[2 * i % 8] | uint32_t(v[(2 * i + 1) % 8]) << 16;
        }
    }
    __device__ __forceinline__ void store(void *row, uint32_t unit, uint32_t dim) const
    {
        if constexpr (!SPREAD && T::words == 8) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<char *>(row) + unit * bytes), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                         "r"(w[5]), "r"(w[6]), "r"(w[7])
                         : "memory");
        } else if constexpr (!SPREAD) {
            uint4 *p = reinterpret_cast<uint4 *>(static_cast<char *>(row) + unit * bytes);
#pragma unroll
            for (int i = 0; i < T::words / 4; i++) p[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else {
            using E = std::conditional_t<T::words == 8, uint32_t, uint16_t>;
            const uint32_t first = column_of<true>(unit, 0);
            E *p = static_cast<E *>(row) + first, v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = E(T::words == 8 ? w[i % T::words] : i & 1 ? w[i / 2] >> 16 : w[i / 2]);
            if ((unit & ~31u) * 8 + 256 <= dim) {
#pragma unroll
                for (int i = 0; i < 8; i++) p[32 * i] = v[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (first + 32 * i < dim) p[32 * i] = v[i];
            }
        }
    }
    __device__ __forceinline__ void get(Pair (&f)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (T::words == 8) {
                f[i] = pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            } else if constexpr (std::is_same_v<T, B16>) {
                f[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
            } else {
                const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                f[i] = pair(v.x, v.y);
            }
        }
    }
    __device__ __forceinline__ void set(const Pair (&f)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 v = both(f[i]);
            if constexpr (T::words == 8) w[2 * i] = __float_as_uint(v.x), w[2 * i + 1] = __float_as_uint(v.y);
            else if constexpr (std::is_same_v<T, B16>) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v.y), "f"(v.x));
            else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v.y), "f"(v.x));
        }
    }
};

// The 128 random bits of 8 columns of a row.
__device__ __forceinline__ uint4 random_bits(const DropKeys &d, uint32_t unit, uint32_t row)
{
    uint32_t a = unit, b = row, c = d.offset0, e = d.offset1;
#pragma unroll
    for (int i = 0; i < kRounds; i++) {
        const uint64_t x = uint64_t(0xD2511F53u) * a, y = uint64_t(0xCD9E8D57u) * c;
        a = uint32_t(y >> 32) ^ b ^ d.key[2 * i];
        b = uint32_t(y);
        c = uint32_t(x >> 32) ^ e ^ d.key[2 * i + 1];
        e = uint32_t(x);
    }
    return make_uint4(a, b, c, e);
}

// Dropout of a unit's values.  SPREAD: the warp's 32 units of random bits lie in shared memory until the lanes have taken theirs.
template <bool SPREAD> __device__ __forceinline__ void drop_values(const DropKeys &d, uint4 *bits, uint32_t unit, uint32_t row, Pair (&x)[4])
{
    const uint4 r = random_bits(d, unit, row + d.first);
    const Pair keep = pair(d.keep, d.keep);
    if constexpr (!SPREAD) {
        // a half of a word reaches the border where the word, with that half on top, reaches border << 16
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 v = both(mul2(x[i], keep));
            x[i] = pair(w[i] << 16 >= d.border16 ? v.x : 0.0f, w[i] >= d.border16 ? v.y : 0.0f);
        }
    } else {
        const uint32_t lane = threadIdx.x & 31;
        __syncwarp();
        bits[lane] = r;
        __syncwarp();
        const uint16_t *of = reinterpret_cast<const uint16_t *>(bits) + lane;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 v = both(mul2(x[i], keep));
            x[i] = pair(of[64 * i] >= d.border ? v.x : 0.0f, of[64 * i + 32] >= d.border ? v.y : 0.0f);
        }
    }
}

// ------------------------------------------------------------------------------------------------ sums over a row

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// The larger one; NaN where either is (fmaxf would drop it).
__device__ __forceinline__ float max_nan(float x, float y)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}

// The largest magnitude of most and two values at once.
__device__ __forceinline__ float most_of(float most, float2 v)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(most), "f"(v.x), "f"(v.y));
    return r;
}

struct Meeting {
    float2 of_warp[2][kWarps];
    float2 of_block[2][8];
};

// Before the first meeting of a row's thread blocks: nobody writes to a block's shared memory until that block has begun.  Said first and
// waited for after the first rows have been asked for, which lie in a block's own.
__device__ __forceinline__ void cluster_begins(uint32_t blocks)
{
    if (blocks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_has_begun(uint32_t blocks)
{
    if (blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// (sum, maximum of what is not negative, NaN where one is) over the threads of a row: a warp, or `blocks` thread blocks of a cluster.  Two sets of places
// take turns: whoever writes to one has seen every thread arrive after its last reading.
template <bool WARP> __device__ __forceinline__ float2 join_row(float2 v, bool want_most, Meeting &m, uint32_t turn, uint32_t blocks, uint32_t rank)
{
#pragma unroll
    for (int d = 16; d; d /= 2) v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
    // the bits of numbers that are not negative are in their order, NaN's (max_nan's, positive) above infinity's
    if (want_most) v.y = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v.y)));
    if (WARP) {
        __syncwarp();
        return v;
    }
    const uint32_t set = turn & 1, warps = blockDim.x / 32;
    if (warps > 1) {
        if ((threadIdx.x & 31) == 0) m.of_warp[set][threadIdx.x >> 5] = v;
        __syncthreads();
        v = m.of_warp[set][0];
        for (uint32_t k = 1; k < warps; k++) {
            const float2 o = m.of_warp[set][k];
            v = make_float2(v.x + o.x, max_nan(v.y, o.y));
        }
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
        v = make_float2(v.x + o.x, max_nan(v.y, o.y));
    }
    return v;
}

// Which rows and which units of them a thread has: unit, unit + step, ...  (`threads`: of the block; `grid`: blocks that have rows.)
// FULL: every thread has every unit it could have.
template <bool SPREAD, bool WARP, bool FULL> struct Place {
    size_t row, rows;         // first row, and how many rows further the next is
    uint32_t unit, step, end, rank;
    __device__ __forceinline__ Place(uint32_t units, uint32_t per_block, uint32_t blocks, uint32_t threads, uint32_t grid)
    {
        uint32_t thread;
        asm volatile("mov.u32 %0, %%tid.x;" : "=r"(thread));        // once
        if (WARP) {
            row = size_t(blockIdx.x) * kWarps + (thread >> 5);
            rows = size_t(grid) * kWarps;
            unit = thread & 31;
            step = 32;
            end = units;
            rank = 0;
        } else {
            rank = blocks > 1 ? cluster_rank() : 0;
            row = blocks > 1 ? blockIdx.x / blocks : blockIdx.x;
            rows = blocks > 1 ? grid / blocks : grid;
            unit = rank * per_block + thread;
            step = threads;
            end = min(units, (rank + 1) * per_block);
        }
    }
    // whether there is a unit k; SPREAD: a warp has the 256 columns of its units together
    __device__ __forceinline__ bool has(int k) const { return FULL || (SPREAD ? (unit + k * step) & ~31u : unit + k * step) < end; }
    __device__ __forceinline__ bool first() const { return rank == 0 && (WARP ? threadIdx.x & 31 : threadIdx.x) == 0; }
};

// ------------------------------------------------------------------------------------------------ rows on their way

// Rows that are made of units come through shared memory: one thread of a row's (a warp has a ring of its own) asks for the rows of the
// next turns by bulk copies, so that they come in while this turn's is worked on.  A stage has the parts of up to three matrices one
// after the other.
extern __shared__ __align__(128) unsigned char ring[];

struct Piece {
    const void *p;
    size_t stride;            // bytes
    uint32_t unit;            // bytes of 8 values
};

template <bool WARP> struct Stream {
    uint32_t full, base, stage, stages, s = 0, parity = 0;
    bool asks, dead = false;
    __device__ __forceinline__ Stream(uint64_t (*bars)[kMostStages], const RowRing &r) : stage(r.stage), stages(r.stages)
    {
        const uint32_t warp = WARP ? threadIdx.x >> 5 : 0;
        full = smem_addr(bars[warp]);
        base = warp * stages * stage;
        asks = (WARP ? threadIdx.x & 31 : threadIdx.x) == 0;
        if (asks) {
            for (uint32_t i = 0; i < stages; i++) bar_init(full + 8 * i, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        if (WARP) __syncwarp();
        else __syncthreads();
    }
    // units unit0.. of a row into stage `to`
    template <int N> __device__ __forceinline__ void ask(uint32_t to, const Piece (&pieces)[N], size_t row, uint32_t unit0, uint32_t units) const
    {
        uint32_t bytes = 0;
#pragma unroll
        for (int i = 0; i < N; i++)
            if (pieces[i].p) bytes += units * pieces[i].unit;
        bar_expect(full + 8 * to, bytes);
        uint32_t dst = smem_addr(ring) + base + to * stage;
#pragma unroll
        for (int i = 0; i < N; i++)
            if (pieces[i].p) {
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                             "l"(static_cast<const char *>(pieces[i].p) + row * pieces[i].stride + size_t(unit0) * pieces[i].unit), "r"(units * pieces[i].unit), "r"(full + 8 * to)
                             : "memory");
                dst += units * pieces[i].unit;
            }
    }
    // The present stage, once it is there.  Who gives up notes it, goes on without data and waits no more: the block's barriers are
    // still met.
    __device__ __forceinline__ const unsigned char *wait()
    {
        if (!dead && !bar_try(full + 8 * s, parity)) {
            const long long t0 = clock64();
            while (!bar_try(full + 8 * s, parity))
                if (clock64() - t0 > kWaitCycles) {
                    atomicExch(&g_wait_status, 1);
                    dead = true;
                    break;
                }
        }
        return ring + base + s * stage;
    }
    __device__ __forceinline__ void advance()
    {
        if (++s == stages) {
            s = 0;
            parity ^= 1;
        }
    }
};

}  // namespace

}  // namespace rd

#endif  // RD_NORM_ROWS_H_
