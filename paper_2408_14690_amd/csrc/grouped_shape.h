// Shape of the tiles of the grouped experts' products.  Host code without HIP, so that a test can ask it.
#pragma once

#include <cmath>

namespace teal {

// Chosen by the rows that an expert has on average (r).  Few rows: what counts is that W is read once and much
// of it at a time, two blocks on a compute unit.  Many: the tiles that load least for what they multiply, as long as
// they fill the units; compared by the rounds of tiles that the units take and the time of a slab (us, measured on
// full launches), the last tile of an expert taken as half empty.  What was measured (us, gate and up / down):
//   bf16, 64 tokens, 2 of 8 experts of 4096 -> 14336 (r = 16)      32 x 128 347 / 185, 64 x 128 348 / 160, 128 x 256 346 / 179
//   256 tokens of the same (r = 64)       64 x 128 444 / 241, 128 x 128 411 / 185, 128 x 256 380 / 214, 256 x 256 413 / 290
//   2048 tokens (r = 512)                 128 x 128 1302 / 695, 128 x 256 998 / 603, 256 x 256 1027 / 744
//   8192 tokens (r = 2048)                128 x 256 3753 / 2040, 256 x 256 3537 / 2043
//   4096 tokens, 8 of 128 experts of 2048 -> 768 (r = 256)         128 x 128 335 / 314, 128 x 256 262 / 260, 256 x 256 276 / 265
//   mx4, where every block converts what it reads, 2 of 8 experts of 4096 -> 14336:
//   r = 4      32 x 128 169 / 90, 64 x 128 slower
//   r = 64     64 x 128 268 / 177, 256 x 128 295 / 145, 256 x 256 291 / 265
//   r = 128    64 x 128 426 / 260, 256 x 128 412 / 231, 256 x 256 400 / 346
//   r = 512    64 x 128 1427 / 754, 256 x 128 1093 / 646, 256 x 256 986 / 751
//   1200 tokens, 6 of 64 experts of 2048 -> 1408 (r = 112)         64 x 128 162 / 107, 256 x 128 195 / 133, 256 x 256 180 / 130
// So mx4 from 8 to 128 rows, which takes 64 x 128 whatever the width, is not always at its best: at r = 64 W_down of few wide
// experts loses 22 % to 256 x 128, at r = 128 gate and up 7 % and W_down 13 %; many small experts of uneven groups (the last
// line) gain 11 and 21 % by it.  The host knows pairs and experts only: pairs without an expert count in r, and so do
// experts without pairs.
struct GroupedShape {
    int bm, bn;          // rows and columns of a tile; of gate and up half the columns are each one's
};
inline GroupedShape grouped_shape(bool mx4, long long pairs, int all_experts, int cols)
{
    const double experts = pairs < all_experts ? (double)pairs : (double)all_experts, r = pairs / experts;
    if (r <= 8) return {32, 128};
    if (r <= (mx4 ? 128 : 32)) return {64, 128};
    auto time = [&](int bm, int bn, double slab) {
        const double tiles = r <= bm / 2 ? experts : experts * (r / bm + 0.5);
        return std::ceil(tiles * ((cols + bn - 1) / bn) / 256) * slab;
    };
    if (mx4) return {256, time(256, 128, 0.96) < time(256, 256, 1.7) ? 128 : 256};
    const double narrow = time(128, 128, 0.65), wide = time(128, 256, 1.0), large = time(256, 256, 1.85);
    if (large < wide && large < narrow) return {256, 256};
    return {128, narrow < wide ? 128 : 256};
}

}  // namespace teal
