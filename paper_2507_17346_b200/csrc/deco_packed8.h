// The layout of activations kept in 8 bits, for the files that read or write it: a row of `cols` entries is
// ceil(cols / 32) blocks, each 32 signed bytes (0 beyond the row's end) and one exponent byte b;
// entry j stands for q_j 2^(b - 127), b = 255 for NaN.  (b = 0, which is never written, reads as a step of 0.)
#pragma once

#include <stdint.h>

namespace deco {

constexpr uint32_t BLOCK8 = 32;

}  // namespace deco
