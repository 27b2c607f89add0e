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
    char *h;                                 /* between the products, rows of h_row bytes.  few: [active][part][token], else [place][part] */
    float *y;                                /* [place][hidden] */
    int *place;                              /* of each choice in the list by experts, or -1 */
    char *rows;                              /* not few: the tokens' rows on 16-byte boundaries, where x has them elsewhere */
    unsigned long long ld_x, ld_gate_up, ld_down, ld_out;    /* bytes */
    uint32_t tokens, hidden, inter, h_row, top_k, experts;
    int first, activation;
    uint32_t x_row;                          /* few: bytes between the tokens' rows in shared memory */
    uint32_t split;                          /* few: CTAs that share columns of the output */
};

/* Bytes sh .. sh + 15 of two vectors in a row, those from `left` on 0. */
__device__ __forceinline__ uint4 shifted(const uint4 &lo, const uint4 &hi, uint32_t sh, int left)
{
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    /* words first, then the bits within them */
    if (sh & 8u) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (sh & 4u) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    const uint32_t bits = (sh & 3u) * 8u;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], bits);
    if (left < 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = left >= 4 * i + 4 ? w[i] : left <= 4 * i ? 0u : w[i] & ((1u << (left - 4 * i) * 8) - 1u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

/* 16 bytes from any element on, zeros from `left` on. */
__device__ __forceinline__ uint4 load_shifted(const char *p, uint32_t left)
{
    const uint32_t sh = (uint32_t)(uintptr_t)p & 15u;
    const uint4 *const q = reinterpret_cast<const uint4 *>(p - sh);
    const uint4 lo = *q;
    uint4 hi = make_uint4(0u, 0u, 0u, 0u);
    if (sh && left > 16u - sh) hi = q[1];
    return shifted(lo, hi, sh, (int)left);
}

__device__ __forceinline__ float activate(float g, int kind)
{
    if (kind == SIFAR_ACT_SILU) return g / (1.0f + expf(-g));
    return 0.5f * g * (1.0f + erff(g * 0.70710678118654752f));
}

/* Element `col` of a row of h: as it is (PARTS 0), or as so many bf16 values, each the nearest to what the ones before leave, in rows
   `low` bytes apart.  The last one is followed by zeros up to the row's end: the second product reads whole vectors. */
template <int PARTS> __device__ __forceinline__ void store_h(const ExpertsArgs &a, char *row, size_t low, uint32_t col, float v)
{
    using T = typename Elem<PARTS ? SIFAR_BF16 : SIFAR_F32>::type;
    const uint32_t last = col + 1 == a.inter ? a.h_row / (uint32_t)sizeof(T) : 0u;
#pragma unroll
    for (int p = 0; p < (PARTS ? PARTS : 1); ++p) {
        T *const to = reinterpret_cast<T *>(row + p * low);
        if constexpr (PARTS) {
            to[col] = narrow<SIFAR_BF16>(v);
            v -= widen<SIFAR_BF16>(narrow<SIFAR_BF16>(v));
        } else {
            to[col] = narrow<SIFAR_F32>(v);
        }
        for (uint32_t i = a.inter; i < last; ++i) to[i] = (T)0;
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

/* What a CTA works out of the choices: experts that have tokens (list), where each one's tokens begin in the list by experts (first, and
   place by the expert's number), passes of `columns` tokens before each (passes), the tokens by expert in their order (token). */
struct ExpertPlan { int active; uint32_t passes, columns; };

/*
 * A bit per expert and token that chose it (twice: once): an expert's tokens are counted and numbered by bits, in the same order in
 * every CTA.  bits: experts x (tokens / 32) words, sum: a word per warp.  pick(n): the columns of a pass, the same for all threads;
 * n: the tokens of the thread's experts.  `tell`: this CTA writes the places for the sum over a token's choices.  All of the
 * CTA; the barrier behind it is the caller's.
 */
template <int THREADS, typename Pick>
__device__ __forceinline__ ExpertPlan plan_experts(const ExpertsArgs &a, Pick pick, uint32_t *bits, unsigned long long *sum, uint16_t *place, uint16_t *list,
                                                   uint16_t *first, uint16_t *passes, uint8_t *token, bool tell)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const uint32_t words = (a.tokens + 31) / 32, choices = a.tokens * a.top_k;
    for (uint32_t i = threadIdx.x; i < a.experts * words; i += THREADS) bits[i] = 0u;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < choices; i += THREADS) {
        const uint32_t e = local_expert(a, a.indices[i]), t = i / a.top_k;
        if (e < a.experts) atomicOr(&bits[e * words + t / 32], 1u << (t % 32));
    }
    __syncthreads();
    /* in one sum over the experts: how many have tokens, their tokens, their passes */
    constexpr uint32_t kEach = (SIFAR_ROUTE_MAX_EXPERTS + THREADS - 1) / THREADS;
    uint32_t n[kEach];
    unsigned long long mine = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = threadIdx.x * kEach + i;
        n[i] = 0;
        if (e < a.experts)
            for (uint32_t w = 0; w < words; ++w) n[i] += __popc(bits[e * words + w]);
    }
    const uint32_t columns = pick(n);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i)
        mine += (unsigned long long)(n[i] ? 1u : 0u) << 40 | (unsigned long long)n[i] << 20 | (n[i] + columns - 1) / columns;
    unsigned long long upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) sum[warp] = upto;
    __syncthreads();
    unsigned long long before = upto - mine, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += sum[w];
        all += sum[w];
    }
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        if (!n[i]) continue;
        const uint32_t e = threadIdx.x * kEach + i, at = (uint32_t)(before >> 40);
        list[at] = (uint16_t)e;
        place[e] = first[at] = (uint16_t)((before >> 20) & 0xFFFFFu);
        passes[at] = (uint16_t)(before & 0xFFFFFu);
        before += 1ull << 40 | (unsigned long long)n[i] << 20 | (n[i] + columns - 1) / columns;
    }
    const ExpertPlan plan{(int)(all >> 40), (uint32_t)(all & 0xFFFFFu), columns};
    if (threadIdx.x == 0) {
        first[plan.active] = (uint16_t)((all >> 20) & 0xFFFFFu);
        passes[plan.active] = (uint16_t)plan.passes;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < choices; i += THREADS) {
        const uint32_t e = local_expert(a, a.indices[i]), t = i / a.top_k;
        int at = -1;
        if (e < a.experts) {
            at = place[e] + __popc(bits[e * words + t / 32] & ((1u << (t % 32)) - 1u));
            for (uint32_t w = 0; w < t / 32; ++w) at += __popc(bits[e * words + w]);
            token[at] = (uint8_t)t;
        }
        if (tell) a.place[i] = at;
    }
    return plan;
}

/* bf16 rows of whole 16-byte pieces, more tokens than k_up_few takes: the two products, up to k_gather, and `place` for it. */
cudaError_t launch_expert_tiles(cudaStream_t stream, const ExpertsArgs &a);

}  /* namespace sifar */
#endif
