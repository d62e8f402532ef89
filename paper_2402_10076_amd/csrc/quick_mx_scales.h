// Where the tiled products' copies of scales read: plain arithmetic, which the
// kernel and the host's check of it share.
#pragma once
#include <cstdint>

namespace quick {

// A lane's byte offset, which the buffer's size bounds, and the wave's, which
// is added behind that check.
struct BufferPlace {
    uint32_t lane, uniform;
};

// First 16 bytes that a lane copies: of a row's scales (KB a row), or of a
// column tile's packed ones (256 bytes for each four steps; 16 lanes a tile).
constexpr uint32_t row_scales(uint32_t row, int KB) { return row * (uint32_t)KB; }
constexpr uint32_t tile_scales(int tile, int KQ, int lane) { return (uint32_t)tile * KQ * 256 + (lane & 15) * 16; }

// The same of steps 4 q .. 4 q + 3.  A row's last ones may be fewer than four:
// the next row's words after them are not used, and behind the last row there
// are none, so the whole offset is the lane's, for the size to bound.
constexpr BufferPlace scale_copy(uint32_t first, bool rows, int q)
{
    return {first + (uint32_t)q * (rows ? 16u : 256u), 0};
}

}  // namespace quick
