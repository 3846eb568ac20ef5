// Which kernel takes a linear layer on int8 codes (see token_linear.hip), by its sizes.  Host code.  All give the same bits.
#pragma once
#include <algorithm>

namespace mixaq {

enum TokenForm { TOKEN_FEW, TOKEN_MID, TOKEN_SPLIT, TOKEN_TILE, TOKEN_WIDE, TOKEN_LARGE };

// Whether values are quantized on their way into the product: every workgroup does it for its rows
inline bool token_quantized_inside(int x_rows, int KB) { return x_rows <= 16; }

// M rows, KB and NB blocks of 128 inputs and outputs; reach: bytes from the first row of codes that a tile may read to behind the last; values: x is quantized inside
inline TokenForm token_form(int M, int KB, int NB, int experts, bool sorted, long long reach, bool values)
{
    if (values) return TOKEN_FEW;
    const long long rows = sorted ? std::max(1, M / experts) : M, each = (rows + 127) / 128 * NB, tiles128 = sorted ? each * experts : each;
    if (rows <= 32 || tiles128 < 64) return TOKEN_FEW;
    if (reach >= 1LL << 32) return TOKEN_SPLIT;                              // (the tiles count in 32 bits)
    return tiles128 < 1024 ? TOKEN_TILE : TOKEN_LARGE;
}

}  // namespace mixaq
