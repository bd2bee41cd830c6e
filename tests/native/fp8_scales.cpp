// The loads of the scales of the 8-bit products (fp8_scales.h), lane by lane for every
// row count and depth: each reads inside its own row or is far past the buffer, and the
// chunks that a kernel's stages ask for leave every scale in its place before it is used.
#include <cstdio>
#include <vector>

#include "fp8_scales.h"

using namespace oled;

namespace {

constexpr int kNothing = -1;

struct Rows {
  int rows, kb;
  std::vector<int> lds;   // [32][8]: the value of `row * kb + step` held, of one buffer
};

// Byte offset of row r of the item's rows (lanes past the last take it), as the kernels have it.
int row_of(int r, const Rows& x) { return (r < x.rows - 1 ? r : x.rows - 1) * x.kb * 4; }

bool inside(int at, int bytes, int r, const Rows& x) {
  const int lo = row_of(r, x), hi = lo + x.kb * 4;
  if (at >= lo && at + bytes <= hi && hi <= x.rows * x.kb * 4) return true;
  std::printf("rows %d kb %d: row %d bytes [%d, %d) read at %d + %d\n", x.rows, x.kb, r, lo, hi, at, bytes);
  return false;
}

bool fill(Rows& x, int c) {
  const int chunk = scale_chunk(c, x.kb);
  int off[64];   // soff of the kernels
  for (int l = 0; l < 64; ++l) off[l] = row_of(l >> 1, x) + scale_piece(l);
  if (chunk == kWholeChunk) {
    for (int l = 0; l < 64; ++l) {
      const int at = off[l] + 32 * c;
      if (!inside(at, 16, l >> 1, x)) return false;
      for (int b = 0; b < 4; ++b) x.lds[4 * l + b] = at / 4 + b;
    }
  } else if (chunk == kShortChunk) {
    for (int i = 0; i < 4; ++i)
      for (int l = 0; l < 64; ++l) {
        const int src = scale_row_lane(i, l), r = 8 * i + (l >> 3);
        if (src > 63 || off[src] != row_of(r, x)) {
          std::printf("load %d lane %d takes the row of lane %d\n", i, l, src);
          return false;
        }
        const int at = scale_value(off[src], c, x.kb, l);
        if (at == kFarOffset) {
          x.lds[64 * i + l] = kNothing;
          continue;
        }
        if (!inside(at, 4, r, x)) return false;
        x.lds[64 * i + l] = at / 4;
      }
  }
  return true;
}

}  // namespace

int main() {
  for (int rows = 1; rows <= 32; ++rows)
    for (int kb = 1; kb <= 70; ++kb) {
      Rows x{rows, kb, std::vector<int>(256, kNothing)};
      // chunks as the stages ask for them: 0 before the first, c + 1 at stage 8 c
      Rows two[2] = {x, x};
      if (!fill(two[0], 0)) return 1;
      for (int s = 0; s < kb; ++s) {
        if ((s & 7) == 0 && !fill(two[((s >> 3) + 1) & 1], (s >> 3) + 1)) return 1;
        for (int r = 0; r < rows; ++r)
          if (two[(s >> 3) & 1].lds[8 * r + (s & 7)] != r * kb + s) {
            std::printf("rows %d kb %d: scale of row %d step %d is not in place\n", rows, kb, r, s);
            return 1;
          }
      }
    }
  std::puts("ALL OK");
  return 0;
}
