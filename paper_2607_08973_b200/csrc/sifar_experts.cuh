/*
 * What the kernels of the chosen experts' products share: their arguments, which experts and tokens there are, the values between
 * the two products.
 */
#ifndef SIFAR_EXPERTS_CUH
#define SIFAR_EXPERTS_CUH

#include "sifar_norm_shape.cuh"
#include "sifar_ops.cuh"

namespace sifar {

constexpr int kExpertWarps = 8, kExpertThreads = 32 * kExpertWarps;

struct ExpertsArgs {
    const char *x, *gate_up, *down;
    char *out;
    const int *indices;
    const float *weights;
    char *h;                                 /* between the products, rows of h_row bytes.  few: [active][part][token], tiles: [place][part],
                                                else [token][choice][part] */
    float *y;                                /* tiles: [place][hidden], else [token][choice][hidden] */
    int *place;                              /* tiles: of each choice in the list by experts, or -1 */
    unsigned long long ld_x, ld_gate_up, ld_down, ld_out;    /* bytes */
    uint32_t tokens, hidden, inter, h_row, top_k, experts;
    int first, activation;
    uint32_t x_row;                          /* few: bytes between the tokens' rows in shared memory */
};

__device__ __forceinline__ float activate(float g, int kind)
{
    if (kind == SIFAR_ACT_SILU) return g / (1.0f + expf(-g));
    return 0.5f * g * (1.0f + erff(g * 0.70710678118654752f));
}

/* Element `col` of a row of h (and, bf16, of the row with its rest, `low` bytes on).  The last one is followed by zeros up to
   the row's end: the second product reads whole vectors. */
template <int DT> __device__ __forceinline__ void store_h(const ExpertsArgs &a, char *row, size_t low, uint32_t col, float v)
{
    using T = typename Elem<DT>::type;
    const T hi = narrow<DT>(v);
    reinterpret_cast<T *>(row)[col] = hi;
    if constexpr (DT == SIFAR_BF16) reinterpret_cast<T *>(row + low)[col] = narrow<DT>(v - widen<DT>(hi));
    if (col + 1 == a.inter)
        for (uint32_t i = a.inter; i < a.h_row / sizeof(T); ++i) {
            reinterpret_cast<T *>(row)[i] = (T)0;
            if constexpr (DT == SIFAR_BF16) reinterpret_cast<T *>(row + low)[i] = (T)0;
        }
}

/* ------------------------------------------------------------------------ */
/* which experts                                                             */
/* ------------------------------------------------------------------------ */
/* An index as a number of this rank's experts; not below their number where it is another's. */
__device__ __forceinline__ uint32_t local_expert(const ExpertsArgs &a, int index)
{
    return index < a.first ? 0xFFFFFFFFu : (uint32_t)index - (uint32_t)a.first;
}

/* The expert (0 .. experts - 1) that choice i is the token's first one of, or -1: another rank's, or its second. */
__device__ __forceinline__ int expert_of(const ExpertsArgs &a, uint32_t i)
{
    const uint32_t e = local_expert(a, a.indices[i]);
    if (e >= a.experts) return -1;
    for (uint32_t j = i - i % a.top_k; j < i; ++j)
        if (a.indices[j] == a.indices[i]) return -1;
    return (int)e;
}
/* The token's weight for an expert: that of all its choices of it. */
__device__ __forceinline__ float weight_of(const ExpertsArgs &a, uint32_t token, int expert)
{
    const int *const at = a.indices + token * a.top_k;
    const float *const weights = a.weights + token * a.top_k;
    const uint32_t wanted = (uint32_t)expert + (uint32_t)a.first;
    float w = 0.0f;
#pragma unroll 4
    for (uint32_t j = 0; j < a.top_k; ++j)
        if ((uint32_t)at[j] == wanted) w += weights[j];
    return w;
}

/* Keeps the numbers i of 0 .. n - 1 with on(i), in their order: put(place, i).  Returns how many.  All of the CTA, the same for
   all; scratch: kExpertWarps words. */
template <typename On, typename Put>
__device__ __forceinline__ int keep_in_order(uint32_t n, int *scratch, On on, Put put)
{
    int total = 0;
    for (uint32_t i0 = 0; i0 < n; i0 += kExpertThreads) {
        const uint32_t i = i0 + threadIdx.x;
        const bool in = i < n && on(i);
        const uint32_t votes = __ballot_sync(0xFFFFFFFFu, in);
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x / 32] = __popc(votes);
        __syncthreads();
        int before = total;
        for (int w = 0; w < kExpertWarps; ++w) {
            if (w < (int)(threadIdx.x / 32)) before += scratch[w];
            total += scratch[w];
        }
        if (in) put(before + __popc(votes & ((1u << (threadIdx.x & 31)) - 1u)), i);
        __syncthreads();
    }
    return total;
}

/* The experts that have tokens, in their order: list[i] = the i-th one's number; counts[e] = its tokens.  Returns how many. */
__device__ __forceinline__ int list_experts(const ExpertsArgs &a, int *counts, int *list, int *scratch)
{
    for (uint32_t e = threadIdx.x; e < a.experts; e += kExpertThreads) counts[e] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < a.tokens * a.top_k; i += kExpertThreads) {
        const int e = expert_of(a, i);
        if (e >= 0) atomicAdd(&counts[e], 1);
    }
    __syncthreads();
    return keep_in_order(a.experts, scratch, [&](uint32_t e) { return counts[e] > 0; }, [&](int at, uint32_t e) { list[at] = (int)e; });
}

/* bf16 rows of whole 16-byte pieces, more tokens than k_up_few takes: the two products, up to k_gather, and `place` for it. */
cudaError_t launch_expert_tiles(cudaStream_t stream, const ExpertsArgs &a);

}  /* namespace sifar */
#endif
