// Checks of arguments that the operators' entry points share.
#ifndef RD_CHECKS_H_
#define RD_CHECKS_H_

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "rd.h"

namespace rd {

namespace {

constexpr size_t kMostDim = 65536;
constexpr size_t kMostRows = (size_t(1) << 31) - 1024;       // rows and tokens are counted in 32 bits, with room for padding

inline bool is_float(int dtype) { return dtype == RD_FP32 || dtype == RD_BF16 || dtype == RD_FP16; }
inline size_t size_of(int dtype) { return dtype == RD_INT64 || dtype == RD_FP64 ? 8 : dtype == RD_BF16 || dtype == RD_FP16 ? 2 : 4; }
inline bool known(int dtype) { return dtype >= RD_INT32 && dtype <= RD_FP16; }
inline bool aligned(const void *p, size_t to) { return p && reinterpret_cast<uintptr_t>(p) % to == 0; }

// Memory that a call reads or writes: one run of bytes, or rows of `width` bytes that begin `stride` bytes apart.
struct Span {
    uintptr_t begin, end;
    size_t width, stride;     // stride 0: one run
    Span(const void *p, size_t bytes) : begin(reinterpret_cast<uintptr_t>(p)), end(p ? begin + bytes : begin), width(end - begin), stride(0) {}
    Span(const void *p, size_t rows, size_t row_stride, size_t dim, size_t esize) : Span(p, rows ? ((rows - 1) * row_stride + dim) * esize : 0)
    {
        if (p && rows > 1 && row_stride > dim) {
            width = dim * esize;
            stride = row_stride * esize;
        }
    }
    // Spans that lie apart do not meet, nor do columns side by side in rows of the same buffer, which are rows of the same stride (or
    // one run beside such rows).  Rows of different strides are taken to meet when their spans do.
    bool meets(const Span &o) const
    {
        if (begin >= o.end || o.begin >= end) return false;
        if (stride && o.stride && stride != o.stride) return true;
        const size_t s = stride ? stride : o.stride;
        if (!s) return true;
        const size_t at = o.begin >= begin ? (o.begin - begin) % s : (s - (begin - o.begin) % s) % s;       // where o's rows begin in this one's
        return at < width || at + o.width > s;
    }
};

// A matrix's stride: at least a row (0 for an input whose rows are all the same one), and the whole matrix within the address space.
inline bool stride_ok(size_t rows, size_t stride, size_t dim, size_t esize, bool may_repeat = false)
{
    return (stride >= dim || (may_repeat && stride == 0)) && (rows == 0 || stride <= (size_t(1) << 47) / esize / rows);
}

inline int status_of(cudaError_t e) { return e == cudaSuccess ? RD_OK : RD_ERR_CUDA; }

// Whether a written span meets one that is read, or another written one.
template <int W, int R> bool overlap(const Span (&written)[W], const Span (&read)[R])
{
    for (int i = 0; i < W; i++) {
        for (int j = 0; j < R; j++)
            if (written[i].meets(read[j])) return true;
        for (int j = 0; j < i; j++)
            if (written[i].meets(written[j])) return true;
    }
    return false;
}

}  // namespace

}  // namespace rd

#endif  // RD_CHECKS_H_
