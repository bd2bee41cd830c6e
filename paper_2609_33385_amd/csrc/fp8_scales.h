// Where the scales of the 8-bit products are fetched from, for the kernels and for
// the host's check of every address.
//
// A row of blocks has kb scales in a row. They are fetched a chunk of 8 ahead, 32
// bytes a row in LDS. A chunk that a row has whole takes pieces of 16 bytes, two lanes
// a row. The last chunk of a kb that is no multiple of 8 takes single values, 8 lanes
// a row, and its lanes past the row's end ask for kFarOffset, which reads no memory. A
// chunk that does not exist is not fetched. So every address is inside its row, and
// none depends on how the unit bounds one that is partly inside.
#pragma once

namespace oled {

constexpr int kFarOffset = 0x7FFFFFF0;   // past the end of every buffer: reads zeros

enum { kNoChunk = 0, kWholeChunk = 1, kShortChunk = 2 };

constexpr int scale_chunk(int c, int kb) {
  return 8 * c + 8 <= kb ? kWholeChunk : 8 * c < kb ? kShortChunk : kNoChunk;
}

// Whole chunks: lane's piece of row lane / 2 of 32, from the row's first byte.
constexpr int scale_piece(int lane) { return 16 * (lane & 1); }

// Short chunks: load i of 4 takes rows 8 i .. 8 i + 7 of the 32; the lane that holds
// the piece 0 of this lane's row, and this lane's offset from that piece's.
constexpr int scale_row_lane(int i, int lane) { return 16 * i + 2 * (lane >> 3); }
constexpr int scale_value(int row, int c, int kb, int lane) {
  return 8 * c + (lane & 7) < kb ? row + 32 * c + 4 * (lane & 7) : kFarOffset;
}

}  // namespace oled
