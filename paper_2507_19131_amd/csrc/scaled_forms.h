// Which kernel takes a linear layer in 8-bit float (see scaled_linear.hip), by its sizes.  Host code.
#pragma once
#include <algorithm>

namespace mixaq {

// M rows, KB and NB blocks of 128 inputs and outputs; exact: products and sums of 32 bits; ldx: bytes between rows of codes.
//
// Which kernel takes a product: by rows, the layer and how sums are taken, never by x's type or by whether exact sums become codes, so that values
// in and codes out are the same results.  us (graph replays; few / split, or as it says):
//   FEW while its workgroups - 16 rows and 16 outputs each - times their blocks of K stay few, and for up to 16 rows:
//     64 x 1024 x 1024 3.2 / 7.1    128 x 4096 x 1024 7.2 / 16.8    256 x 1024 x 1024 4.9 / 7.2    1001 x 1000 x 333 5.8 / 7.2 |  1024 x 1024 x 1024
//     13.2 / 8.0    512 x 2048 x 2048 22.9 / 11.5    256 x 4096 x 4096 39.5 / 19.1
//   MID, 32 x 32 by eight waves, where SPLIT's 64 x 64 would be fewer than 192 (few / mid / split): 64 x 4096 x 4096 12.1 / 7.8 / 16.9    682 x 3584 x 352
//     13.2 / 11.5 / 17.2    3272 x 7840 x 32 30.5 / 20.4 / 31.0 |  2048 x 1536 x 384 (192) 11.1 (mid) / 10.6    512 x 2048 x 2048 (256) 13.4 / 11.4
//   SPLIT below 96 tiles of 128 x 128, with more than 32 blocks of K below 192, codes out: 1024 x 1024 x 1024 8.9 / 10.9 (tile)    1024 x 4096 x 1024
//     21.4 / 39.3    269 x 5504 x 5984 (141 tiles, 43 blocks) 47.7 / 55.4 |  4704 x 1536 x 384 (111 tiles) 21.8 / 17.6    8192 x 256 x 256 (128) 10.6 / 5.7;
//     bf16 out the same or 5 % to either side at 64
//   LARGE, to bf16, from 192 tiles of 256 x 256 and two blocks of K: 16384 x 512 x 512 (128) 11.3 (tile) / 13.9    2048 x 1024 x 4096 (128)
//     15.4 / 19.0 |  16384 x 768 x 768 (192) 18.7 / 17.4    8192 x 256 x 2048 (256) 14.2 / 12.8    4096 x 2048 x 4096 (256) 43.9 / 34.9; with a
//     GELU, which a second workgroup on the CU hides, from six blocks: 16384 x 384 x 1536 28.4 (tile) / 33.8    100000 x 256 x 1024 108 / 115 |
//     16384 x 1024 x 2048 57.7 / 52.2
//   LARGE, exact sums, from 224 tiles of 256 x 128 and three blocks: 4096 x 4096 x 1024 (128) 42.6 (tile) / 50.9    65536 x 256 x 1024 (two blocks)
//     56.1 / 60.8 |  4704 x 384 x 1536 (228) 10.8 / 10.4    8192 x 1024 x 1024 (256) 22.4 / 19.7    16384 x 1024 x 2048 75.3 / 70.2
enum ScaledForm { SCALED_FEW, SCALED_MID, SCALED_SPLIT, SCALED_TILE, SCALED_LARGE };
inline ScaledForm scaled_form(int M, int KB, int NB, bool gelu, bool exact, long long ldx)
{
    const long long tiles16 = (M + 15LL) / 16 * NB * 8, tiles128 = (M + 127LL) / 128 * NB;
    const long long large = (M + 255LL) / 256 * (exact ? NB : (NB + 1) / 2);
    if (M <= 16 || tiles16 * KB <= std::min(16384, 5000 + 1400 * KB)) return SCALED_FEW;
    if ((M + 63LL) / 64 * NB * 2 < 192) return SCALED_MID;
    if (tiles128 < (KB > 32 ? 192 : 96) || ldx >= (1 << 22)) return SCALED_SPLIT;      // (rows 4 MB apart: the tiles count in 32 bits)
    return large >= (exact ? 224 : 192) && KB >= (exact ? 3 : gelu ? 6 : 2) ? SCALED_LARGE : SCALED_TILE;
}

// Whether values are quantized on their way into FEW's product: every workgroup does it for its 16 rows, so with many workgroups or blocks a launch of
// its own is shorter.  us of the GPU, f32 / bf16 values, in one launch and in two (the second takes the host another 3.5):
//     1 x 1024 x 4096 3.3 / 3.5, 4.8    64 x 1024 x 1024 4.7 / 4.1, 6.0    1 x 4096 x 4096 6.1 / 6.8, 6.1    256 x 1024 x 1024 10.5 / 7.8, 7.9 |
//     16 x 8192 x 1024 17 / 11, 10    1001 x 1000 x 333 21 / 13, 11    64 x 4096 x 4096 33 / 21, 15
inline bool quantized_inside(int M, int KB, int NB)
{
    return scaled_form(M, KB, NB, false, true, 0) == SCALED_FEW && KB <= 32 && (M + 15LL) / 16 * NB * 8 * KB <= 8192;       // (FEW whatever the sums)
}

}  // namespace mixaq
