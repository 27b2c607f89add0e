/*
 * Shared memory of the products for a few tokens, and how many CTAs of them an SM holds: plain C++.
 */
#ifndef SIFAR_EXPERTS_SHAPE_CUH
#define SIFAR_EXPERTS_SHAPE_CUH

#include "sifar_norm_shape.cuh"

namespace sifar {

/* The tokens' rows in shared memory, at most: of up to 8 tokens, two CTAs of 8 warps per SM; of more, where one may have to do. */
constexpr size_t kFewShared = 92 * 1024, kFewMostShared = 180 * 1024;

/* What k_up_few declares itself, for 8 G tokens: sums of 8 warps twice, bits, tokens and list of the experts, a word per warp; the rows
   behind it start on 128 bytes. */
template <int G> constexpr size_t kFewStatic = (2 * 8 * 16 * 8 * (size_t)G * 4 + SIFAR_ROUTE_MAX_EXPERTS * 10 + 8 * 4 + 127) / 128 * 128;

/* CTAs of an SM with `rows` bytes for the tokens' rows.  (16 binary32 tokens of 1408 columns, 8 experts of 512, leave room for one: 45.5 us;
   shares for the two that the registers allow come in two waves, 49.5.) */
template <int G> constexpr unsigned kFewCtas = G <= 2 ? 2 : 1;      /* by registers */
template <int G> constexpr unsigned few_ctas(size_t rows)
{
    return kFewCtas<G> == 2 && 2 * (kFewStatic<G> + rows + kCtaReserved) <= kSmBytes ? 2 : 1;
}

}  /* namespace sifar */
#endif
