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
    uint32_t per_magic;                      /* ceil(2^20 / experts of a group): e / per = e * per_magic >> 20 for e, per < 2^10 */
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

/* l[j] = the rank-order sum of the logits of expert 32 j + lane; -infinity behind the last expert.  The loads of
   several ranks are under way together. */
template <int DT, int NI>
__device__ __forceinline__ void load_logits(float (&l)[NI], const void *const *logits, int P, unsigned long long at, int experts)
{
    using T = typename Elem<DT>::type;
    constexpr int B = NI <= 4 ? 8 : NI <= 8 ? 4 : NI <= 16 ? 2 : 1;
    const int lane = threadIdx.x & 31;
    for (int r0 = 0; r0 < P; r0 += B) {
        T w[B][NI];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (r0 + b >= P) break;
            const T *p = reinterpret_cast<const T *>(static_cast<const char *>(logits[r0 + b]) + at);
#pragma unroll
            for (int j = 0; j < NI; ++j) w[b][j] = j * 32 + lane < experts ? p[j * 32 + lane] : (T)0;
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (r0 + b >= P) break;
#pragma unroll
            for (int j = 0; j < NI; ++j) l[j] = r0 + b == 0 ? widen<DT>(w[b][j]) : __fadd_rn(l[j], widen<DT>(w[b][j]));
        }
    }
#pragma unroll
    for (int j = 0; j < NI; ++j)
        if (j * 32 + lane >= experts) l[j] = -INFINITY;
}

/*
 * Keys: unsigned words that compare as the values do, 0 below all of them.  NaN is as low as -infinity, -0 is 0.
 */
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t u = __float_as_uint(v != v ? -INFINITY : v + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k)
{
    return __uint_as_float(k ^ ((uint32_t)((int32_t)~k >> 31) | 0x80000000u));
}
__device__ __forceinline__ unsigned long long key_of(double v)
{
    const long long u = __double_as_longlong(v != v ? -INFINITY : v + 0.0);
    return (unsigned long long)(u ^ ((u >> 63) | (long long)0x8000000000000000ull));
}

/* Keys of a lane, largest first: Batcher's odd-even merge exchange. */
template <int N> __device__ __forceinline__ void sort_keys(uint32_t (&k)[N])
{
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int q = p; q >= 1; q /= 2)
#pragma unroll
            for (int j = q % p; j + q < N; j += 2 * q)
#pragma unroll
                for (int i = 0; i < (q < N - j - q ? q : N - j - q); ++i)
                    if ((i + j) / (2 * p) == (i + j + q) / (2 * p)) {
                        const uint32_t hi = max(k[i + j], k[i + j + q]), lo = min(k[i + j], k[i + j + q]);
                        k[i + j] = hi;
                        k[i + j + q] = lo;
                    }
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

/* The lanes of a group when a warp looks at all groups: group lane / step, step lanes each. */
__device__ __forceinline__ int lanes_per_group(int groups) { return 32 >> (groups > 1 ? 32 - __clz(groups - 1) : 0); }

/* The value of the lane's group: the largest of `v`'s run, or the sum of its two largest. */
template <typename F> __device__ __forceinline__ F group_value(const F *v, int per, int groups, int step, bool top2)
{
    const int lane = threadIdx.x & 31, g = lane / step;
    F m1 = -INFINITY, m2 = -INFINITY;
    if (g < groups)
        for (int i = lane % step; i < per; i += step) {
            const F x = v[g * per + i];
            m2 = max(m2, min(m1, x));
            m1 = max(m1, x);
        }
    for (int d = step / 2; d > 0; d >>= 1) {
        const F o1 = __shfl_xor_sync(0xFFFFFFFFu, m1, d), o2 = __shfl_xor_sync(0xFFFFFFFFu, m2, d);
        m2 = max(max(m2, o2), min(m1, o1));
        m1 = max(m1, o1);
    }
    if (!top2 || per == 1) return m1;
    const F sum = m1 + m2;
    return sum != sum ? (F)-INFINITY : sum;
}

/* Whether the lane's group is among the best. */
template <typename F> __device__ __forceinline__ bool group_open(F mine, int groups, int step, int top_groups)
{
    const int g = (threadIdx.x & 31) / step;
    int better = 0;
    for (int i = 0; i < groups; ++i) {
        const F o = __shfl_sync(0xFFFFFFFFu, mine, i * step);
        better += (o > mine || (o == mine && i < g)) ? 1 : 0;
    }
    return g < groups && better < top_groups;
}

/*
 * The choice in binary64, from the logits in shared memory: for the tokens of which binary32 cannot tell.
 * Lane i returns choice i.
 */
template <int NI>
__device__ __noinline__ int choose_exactly(const RouteArgs &a, const float *l, double *v, float top)
{
    const int lane = threadIdx.x & 31;
    const bool by_value = a.bias != nullptr, top2 = a.groups > 1 && a.group_score == SIFAR_GROUP_TOP2;
    double total = 1.0;
    if ((by_value || top2) && a.score == SIFAR_SCORE_SOFTMAX) {
        total = 0.0;
        for (int e = lane; e < a.experts; e += 32) total += exp((double)l[e] - (double)top);
        total = warp_sum(total);
    }
    for (int e = lane; e < a.experts; e += 32) {
        double x = (double)l[e];
        if (by_value || top2) {
            x = a.score == SIFAR_SCORE_SIGMOID ? sigmoid(x) : top == -INFINITY ? 0.0 : exp(x - (double)top) / total;
            if (by_value) x += (double)a.bias[e];
        }
        v[e] = lowest(x);
    }
    __syncwarp();
    uint32_t open = 0xFFFFFFFFu;
    int step = 1;
    if (a.groups > 1) {
        step = lanes_per_group(a.groups);
        const double mine = group_value(v, a.experts / a.groups, a.groups, step, top2);
        open = __ballot_sync(0xFFFFFFFFu, group_open(mine, a.groups, step, a.top_groups));
    }
    uint32_t closed = 0u;
#pragma unroll 1
    for (int j = 0; j < NI; ++j) {
        const int e = j * 32 + lane;
        if (e >= a.experts || (a.groups > 1 && !(open >> (e / (a.experts / a.groups)) * step & 1u))) closed |= 1u << j;
    }
    int chosen = 0;
    for (int i = 0; i < a.top_k; ++i) {
        unsigned long long best = 0ull;
        uint32_t be = 0xFFFFFFFFu;
#pragma unroll 1
        for (int j = 0; j < NI; ++j) {
            if (closed >> j & 1u) continue;
            const int e = j * 32 + lane;
            const unsigned long long k = key_of(by_value ? v[e] : (double)l[e]);
            if (k > best) { best = k; be = (uint32_t)e; }
        }
        const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(best >> 32));
        if ((uint32_t)(best >> 32) != hi) be = 0xFFFFFFFFu;
        const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, be != 0xFFFFFFFFu ? (uint32_t)best : 0u);
        if ((uint32_t)best != lo) be = 0xFFFFFFFFu;
        be = __reduce_min_sync(0xFFFFFFFFu, be);
        if ((int)(be & 31u) == lane) closed |= 1u << (be >> 5);
        if (lane == i) chosen = (int)be;
    }
    return chosen;
}

/*
 * The choice goes by keys of binary32 values whose lowest bits are the item's number, so that a key says where it came
 * from and equal values come in the order of the experts.  A lane sorts its keys once; a round then takes the largest
 * head of the 32 lists (one reduction over the warp, one ballot).
 *
 * What binary32 and the cut bits may hide is looked at afterwards: where two neighbours of the chosen, or the last of
 * them and the best that is left, lie closer than the error of both and are not equal by their inputs, the token is
 * chosen again in binary64 (choose_exactly).  Logits that are compared themselves have no error but the cut bits.
 */
template <int DT, int NI>
__global__ void __launch_bounds__(32 * kRouteWarps) k_route(const RouteArgs a)
{
    __shared__ float s_l[kRouteWarps][NI * 32];
    __shared__ double s_v[kRouteWarps][NI * 32];
    grid_let_next_in();
    const int lane = threadIdx.x & 31;
    const unsigned long long token = (unsigned long long)blockIdx.x * kRouteWarps + threadIdx.x / 32;
    grid_wait();
    if (token >= a.tokens) return;
    float l[NI], *const sl = s_l[threadIdx.x / 32];
    double *const sv = s_v[threadIdx.x / 32];
    load_logits<DT, NI>(l, a.logits, a.P, token * a.ld_logits, a.experts);
#pragma unroll
    for (int j = 0; j < NI; ++j) sl[j * 32 + lane] = l[j];

    const bool by_value = a.bias != nullptr, top2 = a.groups > 1 && a.group_score == SIFAR_GROUP_TOP2;
    const bool softmax = a.score == SIFAR_SCORE_SOFTMAX;
    float top = -INFINITY, sum = 1.0f;                    /* of the softmax over all experts */
    if (softmax && (!a.renormalize || by_value || top2)) {
        bool nan = false;
#pragma unroll
        for (int j = 0; j < NI; ++j) { top = fmaxf(top, l[j]); nan = nan || l[j] != l[j]; }
        top = warp_max(top);
        if (__any_sync(0xFFFFFFFFu, nan)) top = NAN;
        if (top != -INFINITY) {
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < NI; ++j) sum += expf(l[j] - top);
            sum = sifar::warp_sum(sum);
        }
    }

    /* what is compared, and its error: `fixed`, and `relative` times its size, both for a pair */
    float v[NI], fixed = 0.0f, relative = 0.0f;
    bool unsure = false;
#pragma unroll
    for (int j = 0; j < NI; ++j) v[j] = l[j];
    if (by_value || top2) {
        if (softmax) {
            /* l - top, expf, the sum's NI + 5 adds, the division: of a score of at most 1 / sum */
            const float inv = top == -INFINITY ? 0.0f : 1.0f / sum;
            fixed = 2.5f * (NI + 16) * 0x1p-24f * inv;
#pragma unroll
            for (int j = 0; j < NI; ++j) v[j] = top == -INFINITY ? 0.0f : __expf(l[j] - top) * inv;
            fixed += 2.5f * 0x1p-21f * inv;               /* ... __expf for expf: two steps and the argument's product */
        } else {
            /* __expf: two steps and the argument's product, |l| exp(-|l|) <= 0.37 steps; the reciprocal: one step */
            fixed = 2.5f * 0x1p-21f;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const float t = __expf(-fabsf(l[j]));
                v[j] = __fdividef(l[j] < 0.0f ? t : 1.0f, 1.0f + t);
            }
        }
        relative = 2.5f * 0x1p-24f + 1.25f * NI * 0x1p-23f;
        if (by_value) {
#pragma unroll
            for (int j = 0; j < NI; ++j)
                if (j * 32 + lane < a.experts) v[j] += a.bias[j * 32 + lane];
        }
        bool nan = false;
#pragma unroll
        for (int j = 0; j < NI; ++j) nan = nan || (j * 32 + lane < a.experts && v[j] != v[j]);
        unsure = __any_sync(0xFFFFFFFFu, nan);
    }
    uint32_t open = 0xFFFFFFFFu;
    int step = 1, per = a.experts;
    if (a.groups > 1) {
        float *const sf = reinterpret_cast<float *>(sv);
#pragma unroll
        for (int j = 0; j < NI; ++j) sf[j * 32 + lane] = v[j] != v[j] ? -INFINITY : v[j];
        __syncwarp();
        step = lanes_per_group(a.groups);
        per = a.experts / a.groups;
        const float mine = group_value(sf, per, a.groups, step, top2);
        const bool in = group_open(mine, a.groups, step, a.top_groups);
        open = __ballot_sync(0xFFFFFFFFu, in);
        if (by_value || top2) {
            const float least = of_key(__reduce_min_sync(0xFFFFFFFFu, in ? key_of(mine) : 0xFFFFFFFFu));
            const float most = of_key(__reduce_max_sync(0xFFFFFFFFu, in || lane / step >= a.groups ? 0u : key_of(mine)));
            /* a sum of two: twice the error, and its own rounding */
            unsure = unsure || !(least - most > 2.0f * fixed + 2.0f * relative * fmaxf(fabsf(least), fabsf(most)));
        }
    }

    const bool logits_decide = !by_value;
    uint32_t key[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const uint32_t e = (uint32_t)(j * 32 + lane);
        key[j] = (key_of(logits_decide ? l[j] : v[j]) & ~(uint32_t)(NI - 1)) | (uint32_t)(NI - 1 - j);
        bool in = e < (uint32_t)a.experts;
        if (a.groups > 1) in = in && (open >> ((e * a.per_magic >> 20) * step) & 1u);
        if (!in) key[j] = 0u;
    }
    if (logits_decide) fixed = relative = 0.0f;
    sort_keys(key);

    int chosen = 0;                                       /* lane i: the i-th choice and its key */
    uint32_t mykey = 0u;
    for (int i = 0; i < a.top_k; ++i) {
        const uint32_t k = __reduce_max_sync(0xFFFFFFFFu, key[0]);
        const int owner = __ffs(__ballot_sync(0xFFFFFFFFu, key[0] == k)) - 1;
        if (lane == i) { mykey = k; chosen = (NI - 1 - (int)(k & (NI - 1))) * 32 + owner; }
        if (lane == owner) {
#pragma unroll
            for (int j = 0; j + 1 < NI; ++j) key[j] = key[j + 1];
            key[NI - 1] = 0u;
        }
    }
    __syncwarp();
    bool mine = lane < a.top_k;
    float logit = mine ? sl[chosen] : 0.0f;
    {
        const float b = by_value && mine ? a.bias[chosen] : 0.0f, x = of_key(mykey & ~(uint32_t)(NI - 1));
        const float nx = __shfl_down_sync(0xFFFFFFFFu, x, 1), nl = __shfl_down_sync(0xFFFFFFFFu, logit, 1);
        const float nb = __shfl_down_sync(0xFFFFFFFFu, b, 1);
        bool far = x - nx > fixed + relative * fmaxf(fabsf(x), fabsf(nx)) || (logit == nl && b == nb);
        /* the last one against what is left, as far as that is equal to it */
        const int last = a.top_k - 1;
        const float ll = __shfl_sync(0xFFFFFFFFu, logit, last), lb = __shfl_sync(0xFFFFFFFFu, b, last);
        const float lx = __shfl_sync(0xFFFFFFFFu, x, last);
        if (lane >= last) far = true;
        unsure = unsure || !__all_sync(0xFFFFFFFFu, far);
        for (int i = 0; !unsure; ++i) {
            const uint32_t k = __reduce_max_sync(0xFFFFFFFFu, key[0]);
            const float rx = of_key(k & ~(uint32_t)(NI - 1));
            if (k == 0u || lx - rx > fixed + relative * fmaxf(fabsf(lx), fabsf(rx))) break;
            const int owner = __ffs(__ballot_sync(0xFFFFFFFFu, key[0] == k)) - 1;
            const int e = (NI - 1 - (int)(k & (NI - 1))) * 32 + owner;
            if (i == 16 || sl[e] != ll || (by_value && a.bias[e] != lb)) unsure = true;
            if (lane == owner) {
#pragma unroll
                for (int j = 0; j + 1 < NI; ++j) key[j] = key[j + 1];
                key[NI - 1] = 0u;
            }
        }
    }
    if (unsure) {
        __syncwarp();
        chosen = choose_exactly<NI>(a, sl, sv, top);
        logit = mine ? sl[chosen] : 0.0f;
    }

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
    const uint32_t per = (uint32_t)(a.experts / a.groups);
    a.per_magic = ((1u << 20) + per - 1u) / per;
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
