// The scale byte of a block of packed latents: plain arithmetic, without device code.
#pragma once

namespace mtla {

// The scale of 32 bf16 numbers whose largest magnitude has the bits `top` (sign cleared): the smallest power of two of which it is
// at most the seven-fold.  6 is the format's largest number, and what lies between 6 and 7 times the scale is off by at most as much as
// what lies between 4 and 6: letting it go saves the other 31 a bit (Gaussian rows: error 0.112 of the row, 0.115 with the scale
// at 6 or at 8).  It stays between 2^-124 and 2^125: everything read back is then a normal number (at 2^126 the largest
// bf16 numbers would go to 4 times that, which is infinite).  Infinities and NaN make the block NaN.
[[gnu::always_inline]] constexpr unsigned packed_scale_of(unsigned top) {
  if (top >= 0x7f80u) return 255u;
  const int s = (int)(top >> 7) - 2 + ((top & 127u) > 96u ? 1 : 0);
  return (unsigned)(s < 3 ? 3 : (s < 252 ? s : 252));
}

}  // namespace mtla
