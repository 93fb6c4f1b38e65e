// The experts' forward product whose rows before the activation leave in 8 bits: the four lanes that have a row's 32 columns agree on
// their step, and what is written of them for the way back is half of the rows in 16 bits.
//
// Bound by the matrix units as the product is without it: 16384 bf16 slots of 32 experts, 1024 x 4096, 257 us a call; with the rows in 16
// bits 246, with none of them 235.  Floats: 16384 slots of 32 experts, 1024 x 4096, 1326 us, rows kept as floats 1323, not kept 1316; 3000 of 7,
// 499 x 777, 46, 46 and 44.
#include "activation.hpp"
#include "kept.hpp"
#include "products.hpp"

namespace nacho {

namespace {

struct KeptRows {
    static constexpr bool kParts = false;
    static constexpr unsigned parts() { return 1; }
    nacho_kept kept;
    template <typename Tile>
    __device__ void end(const ProductArgs &a, const Place &at, v4f (&acc)[Tile::kFragM][Tile::kFragN], char *stage0, char *stage1) const
    {
        typedef typename Tile::type T;
        static_assert(Tile::kTileN % kBlock == 0, "blocks inside a wavefront's columns");
        T *const out = static_cast<T *>(a.out);
        float bias[8];
        bias_of<T, Tile::kTileN / 8>(a, at, bias);
        Tile::template each_row<true>(a, at, acc, stage0, stage1, [&](unsigned m, int n, int width, float (&v)[8]) {
            unsigned most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = e < width ? v[e] + bias[e] : 0.0f;
                most = magnitude(v[e]) > most ? magnitude(v[e]) : most;
            }
            unsigned other = moved<0xb1>(most);
            most = other > most ? other : most;
            other = moved<0x4e>(most);
            most = other > most ? other : most;
            if (width <= 0) return;
            const unsigned exponent = exponent_of(most);
            const float by = steps_per(exponent);
            unsigned codes[2] = {four_codes(v[0], v[1], v[2], v[3], by), four_codes(v[4], v[5], v[6], v[7], by)};
            if (exponent == 255) codes[0] = codes[1] = 0;
            int8_t *to = kept.code + (int64_t)m * kept.ldc + n;
            if (width >= 8) __builtin_memcpy(to, codes, 8);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < width) to[e] = (int8_t)(codes[e / 4] >> (8 * (e % 4)));
            }
            if (lane_id() % 4 == 0) kept.exponent[(int64_t)m * kept.lde + n / kBlock] = (uint8_t)exponent;
            if (a.act != NACHO_ACT_NONE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = activated<T>(v[e], a.act);
            }
            Tile::put(out + (int64_t)m * a.ldo + n, v, width);
        });
    }
};

}  // namespace

hipError_t launch_experts_forward_kept(int dtype, const ProductArgs &a, const nacho_kept &pre, hipStream_t s)
{
    return launch<FORWARD>(dtype, a, KeptRows{pre}, s);
}

}  // namespace nacho
