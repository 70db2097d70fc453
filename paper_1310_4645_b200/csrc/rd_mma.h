// What the matrix products on the tensor cores have in common: waits, copies by TMA, products and accumulators of tcgen05, and on the
// host the maps of the matrices that TMA reads and writes.  For inclusion in one .cu file each: the status word is the file's own.
#ifndef RD_MMA_H_
#define RD_MMA_H_

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "rd_ptx.h"

namespace rd {

namespace {

__device__ int g_wait_status;             // a wait that was given up

// The same barrier in the first thread block of the pair.
template <int CG> __device__ __forceinline__ uint32_t leader_bar(uint32_t bar)
{
    if (CG == 1) return bar;
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
    return r;
}
template <int CG> __device__ __forceinline__ void bar_arrive_leader(uint32_t bar)
{
    if (CG == 1) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
    else asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_bar<CG>(bar)) : "memory");
}
// Waits by a whole warp, whose lanes go on together; false when the wait gave up.  The copies and products are issued by one
// lane, but the loops around them are the warp's: what is the same in every lane then stays in uniform registers, which is where
// the instructions want their operands.  (Loops of a single lane spent some 500 cycles a step on moving them there, as long as the products of the step.)
__device__ __noinline__ bool warp_wait_slow(uint32_t bar, uint32_t parity)
{
    const long long t0 = clock64();
    do {
        if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
    } while (__any_sync(0xffffffffu, clock64() - t0 < kWaitCycles));
    atomicExch(&g_wait_status, 1);
    return false;
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity)
{
    return __all_sync(0xffffffffu, bar_try(bar, parity)) || __all_sync(0xffffffffu, warp_wait_slow(bar, parity));
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t one;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(one));
    return one;
}

template <int CG> __device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint32_t x, uint32_t y, uint32_t bar)
{
    if (CG == 2)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                     "r"(x), "r"(y), "r"(bar)
                     : "memory");
    else asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(y), "r"(bar)
                 : "memory");
}

// Shared-memory operand descriptor, 128-byte swizzle.  Operands with the summed index innermost: rows of 128 bytes, 8 rows
// make a swizzle atom of 1024 bytes (the stride).  Transposed operands: 64 x 64 boxes, each line of 128 bytes holds 64 rows of
// one summed index; 8 lines make an atom (the stride), the next 64 rows begin 8192 bytes further (the leading offset).
__device__ __forceinline__ uint64_t operand(uint32_t addr, bool transposed)
{
    return uint64_t(addr >> 4) | uint64_t(transposed ? 8192 >> 4 : 1) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}

// F8: e4m3 operands, 32 summed indices an instruction; else 16-bit ones, 16.
template <int CG, bool F8 = false> __device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
#define RD_MMA(GROUP, KIND)                                                                             \
    asm volatile(                                                                                       \
        "{\n\t.reg .pred p;\n\t"                                                                        \
        "setp.ne.b32 p, %4, 0;\n\t"                                                                     \
        "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add)) \
        : "memory")
    if constexpr (CG == 2 && F8) RD_MMA("2", "f8f6f4");
    else if constexpr (CG == 2) RD_MMA("2", "f16");
    else if constexpr (F8) RD_MMA("1", "f8f6f4");
    else RD_MMA("1", "f16");
#undef RD_MMA
}
// Arrives, once the products issued so far are done, at the barrier of every thread block that took part.
template <int CG> __device__ __forceinline__ void mma_commit(uint32_t bar)
{
    if (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(uint16_t(3)) : "memory");
    else asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Starts reading 32 columns of a warp's 32 rows; tmem_wait before the values are used.
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
          "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]),
          "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]),
                   "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]),
                   "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 :
                 : "memory");
}

// The same for 16 columns.
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
          "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]),
                   "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}

// Exponentials (the loss's softmax): one instruction, within about 2^-22 of the value and 0 below 2^-126.  That is less than a
// logit's own error moves it, and 32768 of them come with every tile of 128 x 256.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <bool BF16> __device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void tma_store(const CUtensorMap *map, uint32_t src, uint32_t x, uint32_t y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap *map, uint32_t src, uint32_t x, uint32_t y, uint32_t z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
// Adds to what is there; every value is added to by one thread block per launch, so the order of additions is the launches'.
__device__ __forceinline__ void tma_add(const CUtensorMap *map, uint32_t src, uint32_t x, uint32_t y, uint32_t z)
{
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
// 16 bytes of a box of 32 rows of 128 bytes, in the places the 128-byte swizzle gives them.
__device__ __forceinline__ void box_put(uint32_t box, int row, int unit, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box + row * 128 + ((unit ^ (row & 7)) * 16)), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A warp's box: wait until its last contents have left (unless this is the second half of the present ones); then, when it is
// full, make the writes visible to the copy and say whether this lane issues it.
__device__ __forceinline__ void box_wait(int lane, bool second_half)
{
    if (second_half) return;
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}
__device__ __forceinline__ bool box_full(int lane, bool full)
{
    if (!full) return false;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    return lane == 0;
}
// Whether a box of 64 columns of 16 bits from `col` on may be stored by TMA in rows of `dim`: it writes whole words of 16 bytes, and zeros
// beyond the row's end to fill the last, where something else may lie (rows of 14 values, 16 apart: the next 2 were lost).
__device__ __forceinline__ bool box_within(uint32_t col, uint32_t dim) { return dim % 8 == 0 || col + 64 <= dim || col >= dim; }
__device__ __forceinline__ void box_sent() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }

// A position in rows of `wide` places, advanced by a constant number of places without divisions.
struct Cursor {
    uint32_t x, y, wide, dx, dy;
    __device__ __forceinline__ void set(uint32_t at, uint32_t step, uint32_t row)
    {
        wide = row;
        x = at % row;
        y = at / row;
        dx = step % row;
        dy = step / row;
    }
    __device__ __forceinline__ void advance()
    {
        x += dx;
        y += dy;
        if (x >= wide) {
            x -= wide;
            y++;
        }
    }
};

// A ring's stage and the parity of its turn.
struct Turn {
    uint32_t s = 0, parity = 0, stages;
    __device__ __forceinline__ explicit Turn(uint32_t n) : stages(n) {}
    __device__ __forceinline__ void advance()
    {
        if (++s == stages) {
            s = 0;
            parity ^= 1;
        }
    }
};

template <int CG> __device__ __forceinline__ void pair_sync()
{
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

// ------------------------------------------------------------------------------------------------ host

size_t round_up(size_t x, size_t to) { return (x + to - 1) / to * to; }

struct Part {
    char *base;
    size_t at = 0;
    explicit Part(void *p) : base(static_cast<char *>(p)) {}
    template <typename T> T *take(size_t count)
    {
        T *p = reinterpret_cast<T *>(base + at);
        at += round_up(count * sizeof(T), 1024);
        return p;
    }
};

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder()
{
    static std::atomic<EncodeTiled> known{nullptr};
    EncodeTiled f = known.load(std::memory_order_acquire);
    if (!f) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
        f = reinterpret_cast<EncodeTiled>(p);
        known.store(f, std::memory_order_release);
    }
    return f;
}

// dh: `parts` matrices of n x stride fp32 values, written in boxes of 32 x 32.
bool encode_dh(CUtensorMap *map, void *base, size_t stride, size_t n, size_t parts)
{
    const EncodeTiled f = encoder();
    if (!f) return false;
    const cuuint64_t dims[3] = {stride, n, parts}, strides[2] = {stride * 4, n * stride * 4};
    const cuuint32_t box[3] = {32, 32, 1}, one[3] = {1, 1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, base, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A matrix of 16-bit values, `inner` contiguous ones per row, read or written in boxes of 64 values x box_rows rows.
bool encode(CUtensorMap *map, bool bf16, const void *base, size_t inner, size_t rows, size_t stride, uint32_t box_rows)
{
    const EncodeTiled f = encoder();
    if (!f) return false;
    const cuuint64_t dims[2] = {inner, rows}, strides[1] = {stride * 2};
    const cuuint32_t box[2] = {64, box_rows}, one[2] = {1, 1};
    return f(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(base), dims, strides, box, one,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count_of(int device)
{
    static std::atomic<int> known[64];
    if (device < 0 || device >= 64) return 148;
    int n = known[device].load(std::memory_order_relaxed);
    if (!n) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) n = 148;
        known[device].store(n, std::memory_order_relaxed);
    }
    return n;
}

}  // namespace

}  // namespace rd

#endif  // RD_MMA_H_
