/*
 * sifar_route.cu - the choice of experts from P partial router logits, and its backward pass (see sifar.h).
 *
 * A warp per token.  Lane i holds the logits of experts i, i + 32, ...: equal values then compare by (item, lane), the
 * order of the experts.  Everything stays in registers from the loads to the k results.
 */
#include "sifar_ops.cuh"

namespace sifar {

constexpr int kRouteWarps = 4;               /* tokens per CTA */

struct RouteArgs {
    const void *logits[kMaxRanks];
    const float *bias;
    int *indices;
    float *weights;
    unsigned long long tokens, ld_logits;    /* bytes between two tokens */
    float scale;
    int P, experts, top_k, groups, top_groups, group_score, score, renormalize;
};

struct RouteGradArgs {
    const void *logits[kMaxRanks];
    const int *indices;
    const float *dweights;
    void *dlogits;
    unsigned long long tokens, ld_logits, ld_dlogits;
    float scale;
    int P, experts, top_k, score, renormalize;
};

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    return v;
}

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

/* l[j] = the rank-order sum of the logits of expert 32 j + lane; -infinity behind the last expert. */
template <int DT, int NI>
__device__ __forceinline__ void load_logits(float (&l)[NI], const void *const *logits, int P, unsigned long long at, int experts)
{
    using T = typename Elem<DT>::type;
    const int lane = threadIdx.x & 31;
    T w[NI];
    for (int r = 0; r < P; ++r) {
        const T *p = reinterpret_cast<const T *>(static_cast<const char *>(logits[r]) + at);
#pragma unroll
        for (int j = 0; j < NI; ++j) w[j] = j * 32 + lane < experts ? p[j * 32 + lane] : (T)0;
#pragma unroll
        for (int j = 0; j < NI; ++j) l[j] = r == 0 ? widen<DT>(w[j]) : __fadd_rn(l[j], widen<DT>(w[j]));
    }
#pragma unroll
    for (int j = 0; j < NI; ++j)
        if (j * 32 + lane >= experts) l[j] = -INFINITY;
}

__device__ __forceinline__ double lowest(double v) { return v != v ? -INFINITY : v; }

/* Without a step to infinity: exp is taken of -|l| alone. */
__device__ __forceinline__ float sigmoid(float l)
{
    const float t = expf(-fabsf(l));
    return (l < 0.0f ? t : 1.0f) / (1.0f + t);
}

__device__ __forceinline__ double sigmoid(double l)
{
    const double t = exp(-fabs(l));
    return (l < 0.0 ? t : 1.0) / (1.0 + t);
}

/* s / (sum of the chosen s) needs the s only up to a common factor: where all chosen logits are negative they are
   scaled up by exp(-max), so that the ratio does not underflow with them. */
__device__ __forceinline__ float scaled_sigmoid(float l, float max)
{
    return max < 0.0f ? expf(l - max) / (1.0f + expf(l)) : sigmoid(l);
}

template <int DT, int NI>
__global__ void __launch_bounds__(32 * kRouteWarps) k_route(const RouteArgs a)
{
    grid_let_next_in();
    const int lane = threadIdx.x & 31;
    const unsigned long long token = (unsigned long long)blockIdx.x * kRouteWarps + threadIdx.x / 32;
    grid_wait();
    if (token >= a.tokens) return;
    float l[NI];
    load_logits<DT, NI>(l, a.logits, a.P, token * a.ld_logits, a.experts);

    float top = -INFINITY, sum = 0.0f;                    /* of the softmax over all experts */
    const bool whole_softmax = a.score == SIFAR_SCORE_SOFTMAX && (!a.renormalize || a.bias || a.groups > 1);
    if (whole_softmax) {
        bool nan = false;
#pragma unroll
        for (int j = 0; j < NI; ++j) { top = fmaxf(top, l[j]); nan = nan || l[j] != l[j]; }
        top = warp_max(top);
        if (__any_sync(0xFFFFFFFFu, nan)) top = NAN;
#pragma unroll
        for (int j = 0; j < NI; ++j) sum += expf(l[j] - top);
        if (top == -INFINITY) sum = 1.0f;
        else sum = sifar::warp_sum(sum);
    }

    /* what is compared: v in binary64, or the logits */
    double v[NI];
    const bool by_value = a.bias != nullptr, top2 = a.groups > 1 && a.group_score == SIFAR_GROUP_TOP2;
    if (by_value || top2) {
        double total = 0.0;
        if (a.score == SIFAR_SCORE_SOFTMAX) {
#pragma unroll
            for (int j = 0; j < NI; ++j) { v[j] = exp((double)l[j] - (double)top); total += v[j]; }
            total = warp_sum(total);
        }
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            v[j] = a.score == SIFAR_SCORE_SOFTMAX ? (top == -INFINITY ? 0.0 : v[j] / total) : sigmoid((double)l[j]);
            if (by_value && j * 32 + lane < a.experts) v[j] += (double)a.bias[j * 32 + lane];
            v[j] = lowest(v[j]);
        }
    }
    uint32_t closed = 0u;                                 /* bit j: item j cannot be chosen (any more) */
#pragma unroll
    for (int j = 0; j < NI; ++j)
        if (j * 32 + lane >= a.experts) closed |= 1u << j;

    if (a.groups > 1) {
        const int per = a.experts / a.groups;
        double mine = -INFINITY;                          /* lane g: the value of group g */
        for (int g = 0; g < a.groups; ++g) {
            double m1 = -INFINITY, m2 = -INFINITY;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int e = j * 32 + lane;
                if (e >= g * per && e < (g + 1) * per) {
                    const double x = by_value || top2 ? v[j] : lowest((double)l[j]);
                    m2 = fmax(m2, fmin(m1, x));
                    m1 = fmax(m1, x);
                }
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                const double o1 = __shfl_xor_sync(0xFFFFFFFFu, m1, d), o2 = __shfl_xor_sync(0xFFFFFFFFu, m2, d);
                m2 = fmax(fmax(m2, o2), fmin(m1, o1));
                m1 = fmax(m1, o1);
            }
            const double value = top2 && per > 1 ? lowest(m1 + m2) : m1;
            if (lane == g) mine = value;
        }
        int better = 0;
        for (int g = 0; g < a.groups; ++g) {
            const double o = __shfl_sync(0xFFFFFFFFu, mine, g);
            better += (o > mine || (o == mine && g < lane)) ? 1 : 0;
        }
        const uint32_t open = __ballot_sync(0xFFFFFFFFu, lane < a.groups && better < a.top_groups);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int e = j * 32 + lane;
            if (e < a.experts && !(open >> (e / per) & 1u)) closed |= 1u << j;
        }
    }

    int chosen = 0;                                       /* lane i: the i-th choice and its logit */
    float logit = 0.0f;
    for (int i = 0; i < a.top_k; ++i) {
        double best = -INFINITY;
        float bl = 0.0f;
        int be = 0x7FFFFFFF;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const double x = by_value ? v[j] : lowest((double)l[j]);
            if (!(closed >> j & 1u) && (be == 0x7FFFFFFF || x > best)) { best = x; be = j * 32 + lane; bl = l[j]; }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            const double ob = __shfl_xor_sync(0xFFFFFFFFu, best, d);
            const int oe = __shfl_xor_sync(0xFFFFFFFFu, be, d);
            const float ol = __shfl_xor_sync(0xFFFFFFFFu, bl, d);
            if (ob > best || (ob == best && oe < be)) { best = ob; be = oe; bl = ol; }
        }
        if ((be & 31) == lane) closed |= 1u << (be >> 5);
        if (lane == i) { chosen = be; logit = bl; }
    }

    const bool mine = lane < a.top_k;
    float w;
    if (a.renormalize) {
        bool nan = mine && logit != logit;
        float max = warp_max(mine ? logit : -INFINITY);
        if (__any_sync(0xFFFFFFFFu, nan)) max = NAN;
        w = a.score == SIFAR_SCORE_SOFTMAX ? expf(logit - max) : scaled_sigmoid(logit, max);
        if (!mine || max == -INFINITY) w = 0.0f;
        const float total = sifar::warp_sum(w);
        w = max == -INFINITY ? 0.0f : w / total;
    } else if (a.score == SIFAR_SCORE_SOFTMAX) {
        w = top == -INFINITY ? 0.0f : expf(logit - top) / sum;
    } else {
        w = sigmoid(logit);
    }
    if (mine) {
        a.indices[token * a.top_k + lane] = chosen;
        a.weights[token * a.top_k + lane] = a.scale * w;
    }
}

template <int DT, int NI>
__global__ void __launch_bounds__(32 * kRouteWarps) k_route_grad(const RouteGradArgs a)
{
    using T = typename Elem<DT>::type;
    grid_let_next_in();
    const int lane = threadIdx.x & 31;
    const unsigned long long token = (unsigned long long)blockIdx.x * kRouteWarps + threadIdx.x / 32;
    grid_wait();
    if (token >= a.tokens) return;
    T *out = reinterpret_cast<T *>(static_cast<char *>(a.dlogits) + token * a.ld_dlogits);

    int e = lane < a.top_k ? a.indices[token * a.top_k + lane] : -1;
    float d = lane < a.top_k ? a.scale * a.dweights[token * a.top_k + lane] : 0.0f;
    const bool mine = e >= 0 && e < a.experts;
    if (!mine) { e = -1; d = 0.0f; }
    float logit = -INFINITY;
    if (mine) {
        for (int r = 0; r < a.P; ++r) {
            const float x = widen<DT>(reinterpret_cast<const T *>(static_cast<const char *>(a.logits[r]) + token * a.ld_logits)[e]);
            logit = r == 0 ? x : __fadd_rn(logit, x);
        }
    }

    if (a.score == SIFAR_SCORE_SOFTMAX && !a.renormalize) {
        float l[NI], top = -INFINITY, sum = 0.0f;
        load_logits<DT, NI>(l, a.logits, a.P, token * a.ld_logits, a.experts);
        bool nan = false;
#pragma unroll
        for (int j = 0; j < NI; ++j) { top = fmaxf(top, l[j]); nan = nan || l[j] != l[j]; }
        top = warp_max(top);
        if (__any_sync(0xFFFFFFFFu, nan)) top = NAN;
#pragma unroll
        for (int j = 0; j < NI; ++j) { l[j] = top == -INFINITY ? 0.0f : expf(l[j] - top); sum += l[j]; }
        const float inv = top == -INFINITY ? 0.0f : 1.0f / sifar::warp_sum(sum);
        const float along = sifar::warp_sum(mine && top != -INFINITY ? d * (expf(logit - top) * inv) : 0.0f);
        float o[NI];
#pragma unroll
        for (int j = 0; j < NI; ++j) o[j] = -along;
        for (int i = 0; i < a.top_k; ++i) {
            const int oe = __shfl_sync(0xFFFFFFFFu, e, i);
            const float od = __shfl_sync(0xFFFFFFFFu, d, i);
#pragma unroll
            for (int j = 0; j < NI; ++j)
                if (j * 32 + lane == oe) o[j] += od;
        }
#pragma unroll
        for (int j = 0; j < NI; ++j)
            if (j * 32 + lane < a.experts) out[j * 32 + lane] = narrow<DT>(l[j] * inv * o[j]);
        return;
    }

    /* only chosen experts have a gradient */
    float g;
    if (a.renormalize) {
        const bool nan = mine && logit != logit;
        float max = warp_max(mine ? logit : -INFINITY);
        if (__any_sync(0xFFFFFFFFu, nan)) max = NAN;
        float w = a.score == SIFAR_SCORE_SOFTMAX ? expf(logit - max) : scaled_sigmoid(logit, max);
        if (!mine || max == -INFINITY) w = 0.0f;
        const float total = sifar::warp_sum(w);
        w = max == -INFINITY ? 0.0f : w / total;
        g = w * (d - sifar::warp_sum(mine ? d * w : 0.0f));
        if (a.score == SIFAR_SCORE_SIGMOID) g *= sigmoid(-logit);
    } else {
        g = d * sigmoid(logit) * sigmoid(-logit);
    }
    if (!mine) g = 0.0f;
    /* an index that comes more than once: the first of them stores the sum */
    float total = 0.0f;
    bool first = mine;
    for (int i = 0; i < a.top_k; ++i) {
        const int oe = __shfl_sync(0xFFFFFFFFu, e, i);
        const float og = __shfl_sync(0xFFFFFFFFu, g, i);
        if (oe == e) { total += og; first = first && i >= lane; }
    }
#pragma unroll
    for (int j = 0; j < NI; ++j)
        if (j * 32 + lane < a.experts) out[j * 32 + lane] = (T)0;
    __syncwarp();
    if (first) out[e] = narrow<DT>(total);
}

template <int DT>
static cudaError_t launch_route(dim3 grid, cudaStream_t stream, const RouteArgs &a)
{
    const dim3 block(32 * kRouteWarps);
    if (a.experts <= 64) return launch_op(k_route<DT, 2>, grid, block, 1, 0, stream, a);
    if (a.experts <= 128) return launch_op(k_route<DT, 4>, grid, block, 1, 0, stream, a);
    if (a.experts <= 256) return launch_op(k_route<DT, 8>, grid, block, 1, 0, stream, a);
    if (a.experts <= 512) return launch_op(k_route<DT, 16>, grid, block, 1, 0, stream, a);
    return launch_op(k_route<DT, 32>, grid, block, 1, 0, stream, a);
}

template <int DT>
static cudaError_t launch_route_grad(dim3 grid, cudaStream_t stream, const RouteGradArgs &a)
{
    const dim3 block(32 * kRouteWarps);
    if (a.experts <= 64) return launch_op(k_route_grad<DT, 2>, grid, block, 1, 0, stream, a);
    if (a.experts <= 128) return launch_op(k_route_grad<DT, 4>, grid, block, 1, 0, stream, a);
    if (a.experts <= 256) return launch_op(k_route_grad<DT, 8>, grid, block, 1, 0, stream, a);
    if (a.experts <= 512) return launch_op(k_route_grad<DT, 16>, grid, block, 1, 0, stream, a);
    return launch_op(k_route_grad<DT, 32>, grid, block, 1, 0, stream, a);
}

/* What both directions ask of their sizes. */
static int check_sizes(const char *fn, int P, int dtype, size_t tokens, int experts, int top_k, int score, float scale)
{
    if (P < 1 || P > kMaxRanks || (dtype != SIFAR_BF16 && dtype != SIFAR_F32)) {
        set_error("%s: need 1 <= P <= %d and dtype in {0,1}", fn, kMaxRanks);
        return SIFAR_ERR_INVALID;
    }
    if (experts < 1 || experts > SIFAR_ROUTE_MAX_EXPERTS || top_k < 1 || top_k > SIFAR_ROUTE_MAX_TOP_K || top_k > experts ||
        tokens >= kMaxRows) {
        set_error("%s: need 1 <= experts <= %d, 1 <= top_k <= %d and at most the experts, tokens below 2^31", fn,
                  (int)SIFAR_ROUTE_MAX_EXPERTS, (int)SIFAR_ROUTE_MAX_TOP_K);
        return SIFAR_ERR_INVALID;
    }
    if ((score != SIFAR_SCORE_SOFTMAX && score != SIFAR_SCORE_SIGMOID) || !std::isfinite(scale)) {
        set_error("%s: unknown score, or a scale that is not finite", fn);
        return SIFAR_ERR_INVALID;
    }
    return SIFAR_OK;
}

}  /* namespace sifar */

using namespace sifar;

extern "C" int sifar_route(const sifar_route_args *g, void *stream)
{
    static const char *fn = "sifar_route";
    if (!g) { set_error("%s: no argument block", fn); return SIFAR_ERR_INVALID; }
    if (int rc = check_sizes(fn, g->P, g->dtype, g->tokens, g->experts, g->top_k, g->score, g->scale)) return rc;
    if (g->groups < 1 || g->groups > SIFAR_ROUTE_MAX_GROUPS || g->experts % g->groups || g->top_groups < 1 ||
        g->top_groups > g->groups || g->top_k > g->top_groups * (g->experts / g->groups) ||
        (g->group_score != SIFAR_GROUP_MAX && g->group_score != SIFAR_GROUP_TOP2)) {
        set_error("%s: need 1 <= top_groups <= groups <= %d, groups that divide the experts, top_k experts in the chosen "
                  "groups and a known group score", fn, (int)SIFAR_ROUTE_MAX_GROUPS);
        return SIFAR_ERR_INVALID;
    }
    if (g->tokens == 0) return SIFAR_OK;
    if (!g->indices || !g->weights) { set_error("%s: indices and weights are needed", fn); return SIFAR_ERR_INVALID; }
    const size_t es = elem_size(g->dtype), experts = (size_t)g->experts, ld = g->ld_logits ? g->ld_logits : experts;
    const size_t results = g->tokens * (size_t)g->top_k;
    RowArray all[kMaxRanks + 3];
    int n = 0;
    RouteArgs a;
    for (int r = 0; r < kMaxRanks; ++r) {
        a.logits[r] = r < g->P ? g->logits[r] : nullptr;
        if (r >= g->P) continue;
        if (!a.logits[r]) { set_error("%s: logits[%d] is NULL", fn, r); return SIFAR_ERR_INVALID; }
        all[n++] = RowArray{"logits", a.logits[r], g->tokens, experts, ld, es, false};
    }
    all[n++] = RowArray{"bias", g->bias, 1, experts, experts, sizeof(float), false};
    all[n++] = RowArray{"indices", g->indices, 1, results, results, sizeof(int), true};
    all[n++] = RowArray{"weights", g->weights, 1, results, results, sizeof(float), true};
    if (int rc = check_arrays(fn, all, n)) return rc;
    a.bias = g->bias; a.indices = g->indices; a.weights = g->weights;
    a.tokens = g->tokens; a.ld_logits = ld * es; a.scale = g->scale;
    a.P = g->P; a.experts = g->experts; a.top_k = g->top_k;
    a.groups = g->top_groups == g->groups ? 1 : g->groups;       /* all groups stay in: none to choose */
    a.top_groups = g->top_groups; a.group_score = g->group_score;
    a.score = g->score; a.renormalize = g->renormalize != 0;
    const dim3 grid((unsigned)((g->tokens + kRouteWarps - 1) / kRouteWarps));
    const cudaError_t err = g->dtype == SIFAR_BF16 ? launch_route<SIFAR_BF16>(grid, (cudaStream_t)stream, a)
                                                   : launch_route<SIFAR_F32>(grid, (cudaStream_t)stream, a);
    SIFAR_CUDA(err);
    return SIFAR_OK;
}

extern "C" int sifar_route_backward(const sifar_route_grad_args *g, void *stream)
{
    static const char *fn = "sifar_route_backward";
    if (!g) { set_error("%s: no argument block", fn); return SIFAR_ERR_INVALID; }
    if (int rc = check_sizes(fn, g->P, g->dtype, g->tokens, g->experts, g->top_k, g->score, g->scale)) return rc;
    if (g->tokens == 0) return SIFAR_OK;
    if (!g->indices || !g->dweights || !g->dlogits) {
        set_error("%s: indices, dweights and dlogits are needed", fn);
        return SIFAR_ERR_INVALID;
    }
    const size_t es = elem_size(g->dtype), experts = (size_t)g->experts, results = g->tokens * (size_t)g->top_k;
    const size_t ld = g->ld_logits ? g->ld_logits : experts, ldo = g->ld_dlogits ? g->ld_dlogits : experts;
    RowArray all[kMaxRanks + 3];
    int n = 0;
    RouteGradArgs a;
    for (int r = 0; r < kMaxRanks; ++r) {
        a.logits[r] = r < g->P ? g->logits[r] : nullptr;
        if (r >= g->P) continue;
        if (!a.logits[r]) { set_error("%s: logits[%d] is NULL", fn, r); return SIFAR_ERR_INVALID; }
        all[n++] = RowArray{"logits", a.logits[r], g->tokens, experts, ld, es, false};
    }
    all[n++] = RowArray{"indices", g->indices, 1, results, results, sizeof(int), false};
    all[n++] = RowArray{"dweights", g->dweights, 1, results, results, sizeof(float), false};
    all[n++] = RowArray{"dlogits", g->dlogits, g->tokens, experts, ldo, es, true};
    if (int rc = check_arrays(fn, all, n)) return rc;
    a.indices = g->indices; a.dweights = g->dweights; a.dlogits = g->dlogits;
    a.tokens = g->tokens; a.ld_logits = ld * es; a.ld_dlogits = ldo * es; a.scale = g->scale;
    a.P = g->P; a.experts = g->experts; a.top_k = g->top_k; a.score = g->score; a.renormalize = g->renormalize != 0;
    const dim3 grid((unsigned)((g->tokens + kRouteWarps - 1) / kRouteWarps));
    const cudaError_t err = g->dtype == SIFAR_BF16 ? launch_route_grad<SIFAR_BF16>(grid, (cudaStream_t)stream, a)
                                                   : launch_route_grad<SIFAR_F32>(grid, (cudaStream_t)stream, a);
    SIFAR_CUDA(err);
    return SIFAR_OK;
}
