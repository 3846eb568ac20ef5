// Which kernel takes a linear layer on int8 codes (see token_linear.hip), by its sizes.  Host code.  All give the same bits.
#pragma once
#include <algorithm>

namespace mixaq {

enum TokenForm { TOKEN_FEW, TOKEN_MID, TOKEN_SPLIT, TOKEN_TILE, TOKEN_WIDE };

// Whether values of M rows are quantized on their way into FEW's product: every workgroup quantizes its 16 whole rows for itself, so only rows of no more than it holds
// and few workgroups.  us of graph replays, bf16 / f32 values, in one launch and in two (the second takes the host another 3.5 where nothing is captured):
//   (Every wave for its own block of K, which rows sorted by expert had no registers for, took 4.0 and 3.8 for a single row of 1024 x 4096, 6.0 and 7.3 for 32.)
//   512 of 16 outputs: 1 x 1024 x 4096 (256) 4.3 / 5.1, 4.3 / 5.0    64 x 1024 x 1024 (256) 4.5 / 5.7, 4.6 / 6.2    32 x 1024 x 4096 (512) 5.5 / 6.4, 5.5 / 6.4
//     128 x 1024 x 1024 (512) 5.5 / 6.4, 5.5 / 6.4    16 x 1024 x 8192 (512) 5.4 / 6.3, 5.4 / 6.2 |  64 x 1024 x 4096 (1024) 7.9 / 7.9, 7.9 / 7.8
//   Rows sorted by expert, up to 64 in 1024 of 64 outputs (K x N of experts): 16 of 1024 x 2048 of 32 (1024) 7.7 / 7.8, 7.9 / 7.8    64 the same 12.8 / 13.2, 12.9 / 13.4
//     64 of 512 x 1024 of 8 (128) 5.1 / 6.1, 5.0 / 6.0 |  128 of 512 x 1024 of 8 7.6 / 7.3, 7.4 / 7.2    16 of 1024 x 4096 of 128 (8192) 17.8 / 16.3, 17.6 / 16.2
inline bool token_quantized_inside(int M, int K, int NB, int experts, bool sorted)
{
    if (K < 8 || K > 1024) return false;                                     // (rows of fewer than 8 values have no eight to load)
    return sorted ? M <= 64 && M / experts <= 16 && (long long)experts * NB * 2 <= 1024 : (M + 15LL) / 16 * NB * 8 <= 512;
}

// M rows, KB and NB blocks of 128 inputs and outputs; reach: bytes from the first row of codes that a tile may read to behind the last.  us of graph replays, to bf16:
//   FEW, 16 rows by eight waves, 16 outputs, or 64 where those would be over 1024 workgroups.  MID, 32 x 32 by eight waves, where FEW would be over 512 workgroups and
//     MID is no more than 256, of few blocks of K 512 (few / mid): 64 x 1024 x 1024 3.4 / 4.0    32 x 4096 x 4096 7.5 / 7.6    128 x 1024 x 1024 (512) 4.1 / 4.1 |
//     256 x 1024 x 1024 5.6 / 4.2    256 x 4096 x 1024 12.5 / 7.6    512 x 1536 x 384 5.9 / 4.8    256 x 512 x 2048 (MID 512) 4.6 / 4.3 |  512 x 1024 x 1024 (512)
//     5.4 / 5.6    128 x 4096 x 4096 (512) 11.6 / 12.6    1024 x 1536 x 384 (384) 7.1 / 7.7
//   SPLIT, 64 x 64 by four waves, from 192 tiles (few / split): 1024 x 1536 x 384 (96) 7.1 / 8.6    512 x 4096 x 1024 (128) 12.4 / 14.1 |  2048 x 1536 x 384 (192) 10.3 / 9.2
//     1024 x 1024 x 1024 (256) 9.0 / 7.1    4096 x 256 x 256 (256) 5.9 / 5.2    1024 x 4096 x 1024 (256) 22.2 / 14.7
//   TILE, 128 x 128, from 96 tiles (split / tile): 1024 x 4096 x 1024 (64) 14.7 / 21.3    4096 x 256 x 256 (64) 5.2 / 5.8 |  1024 x 384 x 1536 (96) 6.8 / 6.7
//     4096 x 1536 x 384 (96) 13.6 / 11.1    512 x 4096 x 4096 (128) 24.3 / 21.8    8192 x 256 x 256 (128) 6.3 / 6.3
//   WIDE, 128 x 256, from 256 tiles and two blocks of K, of more than one block of outputs (tile / wide): 4096 x 384 x 1536 (192) 9.3 / 10.2    68208 x 96 x 384 (one block
//     of K) 21.7 / 23.8    68208 x 384 x 96 17.1 / 22.9 |  4096 x 512 x 2048 (256) 11.3 / 11.7    8192 x 1024 x 1024 (256) 16.8 / 16.1    17000 x 192 x 768 (399) 15.1 / 14.1
//     8192 x 4096 x 1024 (256) 43 / 36    16384 x 4096 x 4096 325 / 255
// Rows sorted by expert (the average expert stands for all): FEW up to 16 rows an expert, where a workgroup takes all rows of its expert, else tiles (few / tile / wide,
// 1024 x 2048, 32 experts): 16 rows in all 5.6 / 10.3 / 13.1    256 14.4 / 16.9 / 18.2    512 16.7 / 17.2 / 18.3 |  1024 26.1 / 18.5 / 18.8    4096 74 / 28.5 / 25.7
//   That holds for experts about as busy as one another; a workgroup of FEW takes its expert's tiles one after the other, however many.  1024 rows of 64 experts, few / tile: as
//   many each 24.6 / 29.4, drawn by an uneven router 29.7 / 29.1, all to two 68.5 / 11.0, all to one 129 / 10.9.  The offsets are not known where the choice is made.
//   SPLIT takes all rows of its expert in turn as well: 1048512 rows of 8 experts x 4096 x 1024 4.3 ms in WIDE, 1048640, which reach beyond 2^32 bytes, 27.4 in SPLIT
inline TokenForm token_form(int M, int KB, int NB, int experts, bool sorted, long long reach)
{
    const long long rows = sorted ? M / experts : M, many = sorted ? experts : 1;
    if (rows <= 16) return TOKEN_FEW;
    auto tiles = [&](int side) { return (rows + side - 1) / side * many * NB * (128 / side); };
    if (!sorted) {
        if (tiles(16) <= 512) return TOKEN_FEW;
        if (tiles(32) <= (KB <= 4 ? 512 : 256)) return TOKEN_MID;
        if (tiles(64) < 192) return TOKEN_FEW;
        if (tiles(128) < 96) return TOKEN_SPLIT;
    }
    if (reach >= 1LL << 32) return TOKEN_SPLIT;                              // (the tiles count in 32 bits)
    return NB > 1 && KB > 1 && (rows + 127) / 128 * many * ((NB + 1) / 2) >= 256 ? TOKEN_WIDE : TOKEN_TILE;
}

}  // namespace mixaq
