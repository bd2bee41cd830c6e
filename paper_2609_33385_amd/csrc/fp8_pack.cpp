// Packing of one expert's weights into its 8-bit block (host, at load).
#include <cmath>
#include <cstdint>
#include <cstring>

#include "kernels.h"
#include "oled.h"

namespace {

float from_bf16(uint16_t v) {
  const uint32_t u = static_cast<uint32_t>(v) << 16;
  float f;
  std::memcpy(&f, &u, 4);
  return f;
}

// Nearest e4m3 (ties to even) of |v| <= 448 (what a scale of amax / 448 leaves).
uint8_t to_e4m3(float v) {
  if (std::isnan(v)) return 0x7F;
  const uint8_t sign = std::signbit(v) ? 0x80 : 0;
  const float m = std::fabs(v);
  if (m < 0.015625f) {   // below 2^-6: multiples of 2^-9
    return sign | static_cast<uint8_t>(std::nearbyint(m * 512.f));
  }
  uint32_t u;
  std::memcpy(&u, &m, 4);
  u += 0x7FFFFu + ((u >> 20) & 1u);   // keep 3 bits of the mantissa
  const uint32_t code = (((u >> 23) - 120u) << 3) | ((u >> 20) & 7u);
  return sign | static_cast<uint8_t>(code > 0x7Eu ? 0x7Eu : code);
}

// Quantises a rows x cols matrix in 128 x 128 blocks.
template <class Get>
void pack(int rows, int cols, Get&& get, uint8_t* q, float* scale) {
  for (int rb = 0; rb < rows / 128; ++rb)
    for (int cb = 0; cb < cols / 128; ++cb) {
      float amax = 0.f;
      for (int r = 128 * rb; r < 128 * rb + 128; ++r)
        for (int c = 128 * cb; c < 128 * cb + 128; ++c)
          amax = std::fmax(amax, std::fabs(get(static_cast<size_t>(r) * cols + c)));
      const float s = std::fmax(amax, 0x1p-100f) / 448.f;
      scale[static_cast<size_t>(rb) * (cols / 128) + cb] = s;
      for (int r = 128 * rb; r < 128 * rb + 128; ++r)
        for (int c = 128 * cb; c < 128 * cb + 128; ++c) {
          const size_t i = static_cast<size_t>(r) * cols + c;
          q[i] = to_e4m3(get(i) / s);
        }
    }
}

bool supported(int n) { return n >= 128 && n <= 16384 && n % 128 == 0; }

}  // namespace

extern "C" size_t oled_fp8_expert_bytes(int32_t hidden, int32_t inter) {
  if (!supported(hidden) || !supported(inter)) return 0;
  const size_t n = static_cast<size_t>(hidden) * inter;
  return (3 * n + 12 * (n / 16384) + 255) / 256 * 256;
}

extern "C" oled_status oled_fp8_pack_expert(int32_t dtype, int32_t hidden, int32_t inter,
                                            const void* w13, const void* w2, void* block_out) {
  if (!w13 || !w2 || !block_out || (dtype != OLED_F32 && dtype != OLED_BF16)) {
    oled::set_noctx_error("oled_fp8_pack_expert: NULL weights or block, or bad dtype");
    return OLED_ERR_INVALID_ARG;
  }
  if (!supported(hidden) || !supported(inter)) {
    oled::set_noctx_error("oled_fp8_pack_expert: H and I must be multiples of 128 up to 16384");
    return OLED_ERR_UNSUPPORTED;
  }
  const size_t HI = static_cast<size_t>(hidden) * inter;
  uint8_t* q = static_cast<uint8_t*>(block_out);
  float* s = reinterpret_cast<float*>(q + 3 * HI);
  std::memset(q + 3 * HI, 0, oled_fp8_expert_bytes(hidden, inter) - 3 * HI);
  auto both = [&](const void* w, int rows, int cols, uint8_t* to, float* scale) {
    if (dtype == OLED_F32)
      pack(rows, cols, [&](size_t i) { return static_cast<const float*>(w)[i]; }, to, scale);
    else
      pack(rows, cols, [&](size_t i) { return from_bf16(static_cast<const uint16_t*>(w)[i]); }, to,
           scale);
  };
  both(w13, 2 * inter, hidden, q, s);
  both(w2, hidden, inter, q + 2 * HI, s + 2 * (HI / 16384));
  return OLED_OK;
}
