// Shared memory of the vocabulary operators' matrix products: the ring of stages that the operands come in through, and the boxes
// that results leave through.  Nothing here needs CUDA, so that the bounds can be checked on the host.
#ifndef RD_RING_H_
#define RD_RING_H_

#include <cstdint>

namespace rd {

enum { kStats = 0, kDlogits = 1, kGrads = 2 };

constexpr int kTileN = 256;
constexpr int kTileK = 64;                // 128 bytes: one swizzle span
constexpr int kEpilogueWarps = 8;
// CG thread blocks (one, or a pair) compute a tile of 128 * CG x 256 together: each has 128 rows of the left operand and of the
// accumulators, and 256 / CG rows of the right operand.
constexpr int kRowsM = 128;
// Results leave through one box of 4 KB per epilogue warp, except the softmax statistics, which have the room for another stage.
constexpr uint32_t kBox = 4096;
constexpr uint32_t kMostStages = 16;      // logits with small tiles have more stages in the same room
template <int KIND, int CG> struct Shape {
    static constexpr int tile_m = kRowsM * CG, rows_n = kTileN / CG;
    static constexpr uint32_t stage_a = kRowsM * kTileK * 2, stage_b = rows_n * kTileK * 2, stage = stage_a + stage_b;
    static constexpr int stages = CG == 1 ? 4 : KIND == kStats ? 7 : 6;
    static constexpr uint32_t boxes = KIND == kStats ? 0 : kEpilogueWarps * kBox, ring = stages * stage, smem = ring + boxes + 1024 + 512;
};

// The ring of a logits kernel, whose stages hold a_rows rows of the left operand and columns_n of the right one: as many stages as
// the room holds.  A product reads kRowsM rows of the left operand from the stage's beginning, whatever a_rows is (the accumulators
// that the rows behind a_rows give are not used), so the last stage begins early enough for those to lie in the room too: of 32 rows
// and 64 columns 16 stages would fit, but the products of the last one would read 4 KB beyond.
struct Ring {
    uint32_t stage, stages;   // bytes of a stage, and how many there are
};
constexpr Ring ring_of(uint32_t room, uint32_t a_rows, uint32_t columns_n)
{
    const uint32_t stage = (a_rows + columns_n) * kTileK * 2, fit = room / stage, inside = (room - kRowsM * kTileK * 2) / stage + 1;
    const uint32_t stages = fit < inside ? fit : inside;
    return Ring{stage, stages < kMostStages ? stages : kMostStages};
}

}  // namespace rd

#endif  // RD_RING_H_
