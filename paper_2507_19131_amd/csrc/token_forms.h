// Which kernel takes a linear layer on int8 codes (see token_linear.hip), by its sizes.  Host code.  All give the same bits.
#pragma once
#include <algorithm>

namespace mixaq {

enum TokenForm { TOKEN_FEW, TOKEN_MID, TOKEN_SPLIT, TOKEN_TILE, TOKEN_WIDE };

// Whether values are quantized on their way into FEW's product: every workgroup looks for the maxima of its 16 whole rows, so only where a wave has one block of K
// and workgroups are few.  us of graph replays, bf16 / f32 values, in one launch and in two (the second takes the host another 3.5):
//     1 x 1024 x 4096 4.0 / 5.0, 3.8 / 5.0    16 x 1024 x 4096 4.5 / 5.7, 5.3 / 5.7    64 x 1024 x 1024 4.5 / 5.7, 5.3 / 6.2 |  32 x 1024 x 4096 6.0 / 6.3,
//     7.3 / 6.4    1 x 4096 x 4096 7.4 / 5.9, 7.2 / 6.0    16 x 4096 x 1024 10.0 / 7.3, 16.0 / 7.3
inline bool token_quantized_inside(int M, int KB, int NB) { return KB <= 8 && (M + 15LL) / 16 * NB * 8 <= 256; }

// M rows, KB and NB blocks of 128 inputs and outputs; reach: bytes from the first row of codes that a tile may read to behind the last; values: x is quantized inside
inline TokenForm token_form(int M, int KB, int NB, int experts, bool sorted, long long reach, bool values)
{
    if (values) return TOKEN_FEW;
    const long long rows = sorted ? std::max(1, M / experts) : M, each = (rows + 127) / 128 * NB, tiles128 = sorted ? each * experts : each;
    if (rows <= 32 || tiles128 < 64) return TOKEN_FEW;
    if (reach >= 1LL << 32) return TOKEN_SPLIT;                              // (the tiles count in 32 bits)
    return tiles128 < 1024 ? TOKEN_TILE : TOKEN_WIDE;
}

}  // namespace mixaq
