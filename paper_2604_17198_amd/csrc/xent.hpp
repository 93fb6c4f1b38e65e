// What the kernels of the cross entropy share.
#pragma once
#include "products.hpp"

namespace nacho {

// For f16: the power of two that brings the largest weight of a row next to 2^15.  The products of a gradient read g times it: the small
// probabilities of most of a vocabulary, under weights of one by the number of rows, would vanish.
__device__ inline int scale_exponent(float most)
{
    const int e = most > 0.0f && most < kInfinity ? 14 - ilogbf(most) : 0;
    return e < 100 ? e : 100;
}

// The stretches of the vocabulary by which the rows' gradients are summed.  Where fewer rows count than there are, what is launched and the
// room for the sums hold more stretches of fewer rows.  (Loss and gradients, us so and with the stretches of all rows: 1213 of 2021 rows,
// 100003 x 1024 f16 1209 and 1271; 614 of 2048, 32000 x 1024 bf16 279 and 305; 500 of 1000, 32000 x 512 f32 641 and 777.)
struct Stretches {
    int32_t most, k_part, tall, words, shortest;       // of all rows; tile height; words of a piece; words of a stretch at least
    int64_t rows;
    // Words of a stretch for `live` > 0 rows.
    __device__ int of(int live) const
    {
        const int64_t by_tiles = most * ((rows + tall - 1) / tall) / (((int64_t)live + tall - 1) / tall), by_room = most * rows / live;
        const int64_t by_words = (words + shortest - 1) / shortest, n = by_tiles < by_room ? by_tiles : by_room;
        const int held = (int)(n < by_words ? n : by_words);
        return held <= most ? k_part : ((words + held - 1) / held + 127) / 128 * 128;
    }
};

}  // namespace nacho
