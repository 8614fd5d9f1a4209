// Which calls multiply compressed experts as they are decoded (zipmoe_product.h) and which decode them first: sizes only, host code only.
#pragma once
#include <cstdint>

namespace zipmoe {

constexpr int kProductPairs = 64, kProductVectors = 8;           // most pairs of a call, most vectors that one matrix meets
constexpr uint32_t kProductRows = 4, kProductStream = 8192;      // most matrix rows and values of a stream

// The piece of row r that lies in stream g has number g + r: both grow by one where either changes.  Most rows that a stream touches:
inline uint32_t product_rows(uint32_t width, uint32_t stream_values)
{
    return stream_values % width == 0 ? stream_values / width : width % stream_values == 0 ? 1u : stream_values / width + 2u;
}

// Whether the products can be had at all.
inline bool product_fits(uint32_t hidden, uint32_t intermediate, uint32_t stream_values, int64_t n_tokens, uint64_t pairs)
{
    return n_tokens <= kProductVectors && pairs <= kProductPairs && hidden % 8 == 0 && intermediate % 8 == 0 && stream_values <= kProductStream &&
           product_rows(hidden, stream_values) <= kProductRows && product_rows(intermediate, stream_values) <= kProductRows;
}

// Whether they are ahead of a decode and a product that reads it.  A tile is multiplied with every vector that its expert meets, so the more tokens an
// expert has, the more a product costs that comes with the decode, and the less one that reads each matrix once for all of them; a wave's sums grow with the rows
// of its stream, and with eight vectors they do not fit into the registers (the tiles of one straight group, 4096 values, bear that best, long codes least); a short
// stream has its sums added up over the wave after a few tiles.  us decoded first / multiplied while decoding; p: pairs per named expert, 1 for one token:
//   streams of 512     2048 x 1024, 1 token 55.7 / 58.8; 3 tokens p 1.3 126 / 167
//   streams of 1024    2048 x 1024, 1 token 54.4 / 41.6; 2 tokens p 2.0 53.7 / 52.5; 4 tokens p 2.3 99.9 / 94.0, p 4.0 60.5 / 68.8; 5 tokens p 2.2 132 / 172
//   streams of 2048    2048 x 2048, 1 token 49.6 / 34.2; 4 tokens p 1.2 177 / 101, p 4.0 58.2 / 50.4; 6 tokens p 1.7 191 / 210, 8 tokens p 3.6 127 / 162
//   streams of 4096    2048 x 1024, 1 token 53.6 / 33.6; 4 tokens p 1.8 123 / 80.6, p 4.0 60.0 / 57.3; 8 tokens p 2.8 166 / 124, p 4.3 110 / 102, p 8.0 65 / 91
//     long codes       2048 x 1024, 1 token 56.4 / 41.7; 4 tokens p 4.0 62.6 / 60.9; 8 tokens p 2.8 174 / 165, p 4.3 115 / 124, p 8.0 67.7 / 110
//     eight rows       1376 x 1368, 1 token 31.9 / 23.3; 4 tokens p 1.6 62.4 / 49.1, p 4.0 33.4 / 37.4; 8 tokens p 2.7 76.0 / 77.5, p 3.6 64.0 / 73.8
//     both             1376 x 1368, 1 token 34.7 / 27.9; 4 tokens p 1.6 65.5 / 57.1, p 4.0 36.5 / 42.8; 5 tokens p 1.7 81.6 / 86.3, 8 tokens p 2.7 80.4 / 96.8
//     one row          4096 x 4096, 1 token 91.0 / 42.2; 4 tokens p 4.0 109 / 92.1; 8 tokens p 4.0 220 / 194, p 8.0 113 / 149
//   streams of 8192    4096 x 2048, 1 token 49.4 / 37.0; 4 tokens p 4.0 58.3 / 50.4; 5 tokens p 1.3 221 / 262, 8 tokens p 2.3 198 / 286
//     long codes       4096 x 2048, 1 token 52.8 / 51.0; 4 tokens p 2.0 112 / 94.0, p 4.0 61.5 / 73.8
inline bool product_pays(uint32_t hidden, uint32_t intermediate, uint32_t stream_values, bool long_codes, int64_t n_tokens, uint64_t pairs, uint64_t named)
{
    if (stream_values < 1024) return false;
    const bool many_rows = product_rows(hidden, stream_values) + product_rows(intermediate, stream_values) > 6;
    if (n_tokens > 4 && (stream_values != 4096 || (many_rows && long_codes))) return false;
    // twice the pairs per named expert
    return 2 * pairs <= named * (stream_values < 2048 || many_rows || (stream_values > 4096 && long_codes) ? 5 : 8);
}

}  // namespace zipmoe
