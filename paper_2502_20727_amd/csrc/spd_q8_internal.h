// Packed 8-bit weights as the packers write them and the kernels read them.
#pragma once

#include "spd_internal.h"
#include "spd_q8.h"

// The scales of the N columns, fp32, padded to whole n-tiles; then 1 KiB fragments [n-tile of 16 columns][k-tile of 64 inputs]: the
// register order of the 16 x 16 x 64 MFMA on 8-bit integers, lane 16 g + r holding the 16 inputs 16 g .. of column r.  Zeros
// where K or N end.
SPD_HD int spd_q8_ktiles(int K) { return (K + 63) / 64; }
SPD_HD int spd_q8_ntiles(int N) { return (N + 15) / 16; }
SPD_HD size_t spd_q8_weights_at(int N) { return ((size_t)spd_q8_ntiles(N) * 64 + 255) & ~(size_t)255; }
