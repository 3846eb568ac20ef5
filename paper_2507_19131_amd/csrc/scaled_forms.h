// Which kernel takes a linear layer in 8-bit float (see scaled_linear.hip), by its sizes.  Host code.
#pragma once
#include <algorithm>

namespace mixaq {

// M rows, KB and NB blocks of 128 inputs and outputs; exact: products and sums of 32 bits; ldx: bytes between rows of codes.
//
// Which kernel takes a product: by rows, the layer and how sums are taken, never by x's type or by whether exact sums become codes, so that values
// in and codes out are the same results.  (They go by rows: the same row among more rows may be summed in another order.)  us of graph replays:
//   FEW, 16 rows x 16 outputs by eight waves, while its workgroups times their blocks of K stay few, and for up to 16 rows.  The line lies where FEW and SPLIT
//     meet, at 5000 for a workgroup's start and end and 1400 a block; few / split to bf16: 64 x 1024 x 1024 3.4 / 7.3    128 x 4096 x 1024 7.5 / 17.0
//     256 x 1024 x 1024 5.2 / 7.4    1001 x 1000 x 333 6.0 / 7.4    1024 x 512 x 512 5.1 / 5.9 |  2048 x 512 x 512 8.0 / 6.2    1024 x 1024 x 1024 12.6 / 7.7
//     512 x 2048 x 2048 22.4 / 11.1    256 x 4096 x 4096 38.8 / 17.5.  Of one block of K it is drawn too far (1600 x 128 x 512 5.2 / 4.7    3200 x 128 x 512
//     8.4 / 5.4, tile 4.7), and MID, which came later, is shorter in front of it too (256 x 1024 x 1024 4.3    1001 x 1000 x 333 4.9) but not
//     where workgroups are few (64 x 1024 x 1024 4.1    64 x 8192 x 1024 few 7.4, mid 12.1).  Codes out: FEW's kernel is MID's.
//   MID, 32 x 32 by eight waves, where SPLIT's 64 x 64 would be fewer than 192 (few / mid / split to bf16): 64 x 4096 x 4096 12.2 / 7.9 / 17.2
//     682 x 3584 x 352 11.8 / 10.7 / 15.4 |  2048 x 1536 x 384 (192) 9.5 (mid) / 9.1    512 x 2048 x 2048 (256) 13.2 / 11.1    256 x 4096 x 4096 22.0 / 17.5
//   SPLIT below 96 tiles of 128 x 128, with more than 32 blocks of K below 192 (split / tile; codes out, to bf16 in brackets): 1024 x 1024 x 1024 9.0 / 11.4
//     (7.6 / 8.7)    1024 x 4096 x 1024 21.4 / 33.8 (19.8 / 23.7)    269 x 5504 x 5984 (141 tiles, 43 blocks) 47.7 / 55.4 |  4704 x 1536 x 384 (111 tiles) 19.8 / 15.5
//     (15.5 / 11.4)    8192 x 256 x 256 (128) 10.8 / 6.0 (6.3 / 5.4)
//   LARGE, to bf16, from 192 tiles of 256 x 256 and two blocks of K (tile / large): 16384 x 512 x 512 (128) 11.3 / 13.9    2048 x 1024 x 4096 (128) 15.4 / 19.0
//     8192 x 1024 x 1024 (128) 14.5 / 18.8 |  16384 x 768 x 768 (192) 18.7 / 17.4    8192 x 256 x 2048 (256) 14.2 / 12.8    16384 x 1024 x 2048 49.6 / 41.3; with a
//     GELU, which a second workgroup on the CU hides, from six blocks: 16384 x 384 x 1536 27.0 / 34.1    100000 x 256 x 1024 108 / 115 |
//     16384 x 1024 x 2048 58.6 / 53.0
//   LARGE, exact sums, from 224 tiles of 256 x 128 and three blocks (tile / large, codes out): 4096 x 4096 x 1024 (128) 41.5 / 51.1    65536 x 256 x 1024 (two blocks)
//     56.1 / 60.8 |  4704 x 384 x 1536 (228) 10.5 / 9.9, with a GELU 13.4 / 13.0    8192 x 1024 x 1024 (256) 19.8 / 18.5    16384 x 1024 x 2048 71.8 / 70.6; of three
//     blocks and many tiles the two are alike (16384 x 384 x 1536 26.8 / 26.8, with a GELU 35.0 / 36.8)
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
// its own is shorter.  us of graph replays, f32 / bf16 values, in one launch and in two (the second takes the host another 3.5):
//     1 x 1024 x 4096 3.6 / 3.7, 5.4 / 5.0    64 x 1024 x 1024 5.1 / 4.4, 6.5 / 6.3    1 x 4096 x 4096 6.8 / 7.0, 6.3 / 6.2    256 x 1024 x 1024 11.3 / 8.1,
//     8.9 / 8.2 |  16 x 8192 x 1024 17.9 / 11.2, 10.3 / 10.2    1001 x 1000 x 333 20.6 / 10.9, 11.4 / 10.5
inline bool quantized_inside(int M, int KB, int NB)
{
    return scaled_form(M, KB, NB, false, true, 0) == SCALED_FEW && KB <= 32 && (M + 15LL) / 16 * NB * 8 * KB <= 8192;       // (FEW whatever the sums)
}

}  // namespace mixaq
