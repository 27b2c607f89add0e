/*
 * How rows are laid over threads, CTAs, clusters and blocks of rows, and the shared memory that goes with it: the arithmetic
 * of the norm kernels' launches, plain C++.
 */
#ifndef SIFAR_NORM_SHAPE_CUH
#define SIFAR_NORM_SHAPE_CUH

#include <cstddef>
#include <cstdint>

#include "sifar.h"

namespace sifar {

constexpr unsigned kSms = 148;               /* of a B200 */
constexpr int kMaxRowThreads = 512;
constexpr unsigned kMaxNormCluster = 8;

/* How many CTAs hold a row and how many threads of each. */
struct RowShape {
    unsigned tx, parts;
};
inline RowShape row_shape(int items, size_t cols)          /* items: of a thread */
{
    const size_t need = (cols + items - 1) / items;
    RowShape s;
    for (s.parts = 1;; s.parts *= 2) {
        s.tx = (unsigned)(((need + s.parts - 1) / s.parts + 31) / 32 * 32);
        if (s.tx <= (unsigned)kMaxRowThreads) return s;
    }
}

/* 16 bytes of an array per thread in bf16: with 32 the sums over rows spill (8192 x 4096, two ranks: 107 us against 134;
   two CTAs per SM with 64 registers each: 163). */
template <int DT> constexpr int kGradWords = DT == SIFAR_BF16 ? 4 : 8;

/*
 * Into how many blocks of consecutive rows the rows are cut, and how the blocks lie in CTAs: as many as have room at
 * once, 512 threads per SM (the rows under way and the sums over rows fill its memory and registers).
 */
struct GradShape {
    RowShape row;
    unsigned ry, per_sm;                     /* blocks of a CTA, CTAs of an SM */
    uint32_t blocks;
};

/* Blocks of rows that a B200 holds at once as clusters of `parts` CTAs with `per_sm` CTAs per SM: a row that takes a cluster has 288
   threads of each CTA at least, one CTA per SM (cudaOccupancyMaxActiveClusters: the GPCs do not all have a multiple of 4 SMs). */
inline unsigned clusters_at_once(unsigned parts, unsigned per_sm)
{
    return parts == 1 ? kSms * per_sm : parts == 2 ? kSms / 2 : parts == 4 ? 33 : 15;
}

template <int DT> GradShape grad_shape_of(size_t rows, size_t cols)
{
    const int items = kGradWords<DT> * 4 / (DT == SIFAR_BF16 ? 2 : 4);
    GradShape s;
    s.row = row_shape(items, cols);
    s.ry = s.row.tx == 32 ? 4 : 1;
    s.per_sm = kMaxRowThreads / (s.row.tx * s.ry);
    uint32_t most = clusters_at_once(s.row.parts, s.per_sm) * s.ry;
    /* few rows: a CTA of its own for each */
    while (s.ry > 1 && rows <= most / 2) { s.ry /= 2; most /= 2; }
    s.blocks = (uint32_t)(rows < most ? rows : most);
    return s;
}
inline GradShape grad_shape(int dtype, size_t rows, size_t cols)
{
    return dtype == SIFAR_BF16 ? grad_shape_of<SIFAR_BF16>(rows, cols) : grad_shape_of<SIFAR_F32>(rows, cols);
}

/* What the sums over a row of `values` values take of a CTA's shared memory: a word per warp and a tagged word per CTA of the
   cluster, each twice. */
constexpr size_t row_sum_bytes(int values)
{
    return 2 * (size_t)values * (kMaxRowThreads / 32 * 16 + kMaxNormCluster * 8);
}

/*
 * Shared memory of a CTA for the rows under way: 216 KB of an SM, and no more than leaves room for all CTAs that grad_shape()
 * counts on: each takes its sums and the 1 KB that the system keeps too, in steps of 128 bytes, of 228 KB.  (Nine arrays of 257 to 512
 * bf16 columns, eight CTAs per SM: three stages of 9 KB leave one of the eight out, whose rows come in a second wave.  16384 x 512 of
 * six ranks: 55.6 us so, 43.6 with two stages.)
 */
constexpr uint32_t kMaxStages = 4;
constexpr size_t kSmBytes = 228 * 1024, kCtaReserved = 1024, kRingBytes = 216 * 1024;
constexpr size_t ring_room(unsigned per_sm, int values)
{
    const size_t room = kSmBytes / per_sm / 128 * 128 - kCtaReserved - row_sum_bytes(values), share = kRingBytes / per_sm;
    return room < share ? room : share;
}

/* How many rows of `row_bytes` (all arrays, all threads of a CTA) are under way. */
inline size_t grad_stages(const GradShape &s, size_t rows, size_t row_bytes, int values)
{
    const size_t turns = (rows + s.blocks - 1) / s.blocks;
    size_t stages = ring_room(s.per_sm, values) / row_bytes;
    if (stages > kMaxStages) stages = kMaxStages;
    return stages > turns ? turns : stages;
}

}  /* namespace sifar */
#endif
