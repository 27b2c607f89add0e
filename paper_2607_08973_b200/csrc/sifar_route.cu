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
    int per;                                 /* experts of a group */
    uint32_t per_magic;                      /* ceil(2^20 / per): e / per = e * per_magic >> 20 for e, per < 2^10 */
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

/* Whether the lane's item j is an expert.  NI is the smallest of 2, 4, 8, 16, 32 that holds the experts: from 4 on the
   lower half of the items always is. */
template <int NI> __device__ __forceinline__ bool is_expert(int j, int experts)
{
    return (NI > 2 && j < NI / 2) || j * 32 + (int)(threadIdx.x & 31) < experts;
}

/* l[j] = the rank-order sum of the logits of expert 32 j + lane; -infinity behind the last expert.  The loads of
   several ranks are under way together. */
template <int DT, int NI>
__device__ __forceinline__ void load_logits(float (&l)[NI], const void *const *logits, int P, unsigned long long at, int experts)
{
    using T = typename Elem<DT>::type;
    constexpr int B = NI <= 4 ? 8 : NI <= 8 ? 4 : NI <= 16 ? 2 : 1;
    const int lane = threadIdx.x & 31;
    if (P == 1) {
        const T *p = reinterpret_cast<const T *>(static_cast<const char *>(logits[0]) + at) + lane;
#pragma unroll
        for (int j = 0; j < NI; ++j) l[j] = is_expert<NI>(j, experts) ? widen<DT>(p[j * 32]) : -INFINITY;
        return;
    }
    for (int r0 = 0; r0 < P; r0 += B) {
        T w[B][NI];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (r0 + b >= P) break;
            const T *p = reinterpret_cast<const T *>(static_cast<const char *>(logits[r0 + b]) + at);
#pragma unroll
            for (int j = 0; j < NI; ++j) w[b][j] = is_expert<NI>(j, experts) ? p[j * 32 + lane] : (T)0;
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
        if (!is_expert<NI>(j, experts)) l[j] = -INFINITY;
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

/* One step; 0 of infinity. */
__device__ __forceinline__ float reciprocal(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

/* s / (sum of the chosen s) needs the s only up to a common factor: where all chosen logits are negative they are
   scaled up by exp(-max), so that the ratio does not underflow with them. */
__device__ __forceinline__ float scaled_sigmoid(float l, float max)
{
    return max < 0.0f ? expf(l - max) / (1.0f + expf(l)) : sigmoid(l);
}

/* The lanes of a group when a warp looks at all groups: group lane >> shift, 1 << shift lanes each. */
__device__ __forceinline__ int group_shift(int groups) { return __clz(groups - 1) - 27; }

/* The value of the lane's group: the largest of `v`'s run, or the sum of its two largest. */
template <typename F> __device__ __forceinline__ F group_value(const F *v, int per, int groups, int shift, bool top2)
{
    const int lane = threadIdx.x & 31, g = lane >> shift, step = 1 << shift;
    F m1 = -INFINITY, m2 = -INFINITY;
    const auto look = [&](F x) {
        m2 = max(m2, min(m1, x));
        m1 = max(m1, x);
    };
    const int share = per >> shift;
    if (sizeof(F) == 4 && share << shift == per && (share & 3) == 0) {
        if (g < groups)                                   /* vectors: a lane's share of the group lies side by side */
            for (int i = 0; i < share; i += 4) {
                const float4 q = *reinterpret_cast<const float4 *>(v + lane * share + i);
                look((F)q.x); look((F)q.y); look((F)q.z); look((F)q.w);
            }
    } else if (g < groups) {
#pragma unroll 4
        for (int i = lane & (step - 1); i < per; i += step) look(v[g * per + i]);
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

/* What the choice compares, in binary64. */
__device__ __forceinline__ double value64(const RouteArgs &a, int e, float l, bool scored, double total, float top)
{
    double x = (double)l;
    if (scored) {
        x = a.score == SIFAR_SCORE_SIGMOID ? sigmoid(x) : top == -INFINITY ? 0.0 : exp(x - (double)top) / total;
        if (a.bias) x += (double)a.bias[e];
    }
    return lowest(x);
}

__device__ __noinline__ double softmax_total(const RouteArgs &a, const float *l, float top)
{
    double total = 0.0;
#pragma unroll 4
    for (int e = threadIdx.x & 31; e < a.experts; e += 32) total += exp((double)l[e] - (double)top);
    return warp_sum(total);
}

/* The open groups (bit g) by values in binary64; leaves the values of all experts in v. */
__device__ __noinline__ uint32_t groups_exactly(const RouteArgs &a, const float *l, double *v, float top, double total)
{
    const int lane = threadIdx.x & 31, shift = group_shift(a.groups), g = lane >> shift;
    const bool top2 = a.group_score == SIFAR_GROUP_TOP2;
    __syncwarp();
#pragma unroll 4
    for (int e = lane; e < a.experts; e += 32) v[e] = value64(a, e, l[e], a.bias || top2, total, top);
    __syncwarp();
    const double mine = group_value(v, a.per, a.groups, shift, top2);
    int better = 0;
#pragma unroll 4
    for (int i = 0; i < a.groups; ++i) {
        const double o = __shfl_sync(0xFFFFFFFFu, mine, i << shift);
        better += (o > mine || (o == mine && i < g)) ? 1 : 0;
    }
    return __reduce_or_sync(0xFFFFFFFFu, g < a.groups && better < a.top_groups ? 1u << g : 0u);
}

/* The choice by values in binary64, one expert after the other: lane i returns choice i. */
template <int NI>
__device__ __noinline__ int choose_exactly(const RouteArgs &a, const float *l, double *v, float top, double total, uint32_t open)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
    uint32_t closed = 0u;
#pragma unroll 1
    for (int j = 0; j < NI; ++j) {
        const int e = j * 32 + lane;
        if (e >= a.experts || !(open >> (e / a.per) & 1u)) closed |= 1u << j;
        else v[e] = value64(a, e, l[e], a.bias != nullptr, total, top);
    }
    int chosen = 0;
    for (int i = 0; i < a.top_k; ++i) {
        unsigned long long best = 0ull;
        uint32_t be = 0xFFFFFFFFu;
#pragma unroll 1
        for (int j = 0; j < NI; ++j) {
            if (closed >> j & 1u) continue;
            const int e = j * 32 + lane;                  /* the lane's own value: it stored it */
            const unsigned long long k = key_of(v[e]);
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

/* The candidates e of lanes 0 .. n - 1 in order of their values in binary64: lane i returns the i-th. */
__device__ __noinline__ int order_exactly(const RouteArgs &a, const float *l, int *order, float top, double total, int e, int n)
{
    const int lane = threadIdx.x & 31;
    const double mine = lane < n ? value64(a, e, l[e], a.bias != nullptr, total, top) : 0.0;
    int place = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const double o = __shfl_sync(0xFFFFFFFFu, mine, i);
        const int oe = __shfl_sync(0xFFFFFFFFu, e, i);
        place += (o > mine || (o == mine && oe < e)) ? 1 : 0;
    }
    __syncwarp();
    if (lane < n) order[place] = e;
    __syncwarp();
    return lane < n ? order[lane] : 0;
}

/*
 * The choice goes by keys of binary32 values whose lowest bits are the item's number, so that a key says where it came
 * from and equal values come in the order of the experts.  A lane sorts its keys once; a round then takes the largest
 * head of the 32 lists (one reduction over the warp, one ballot).
 *
 * What binary32 and the cut bits may hide is looked at afterwards: where two neighbours of the chosen, or the last of
 * them and the best that is left, lie closer than the error of both and are not equal by their inputs, rounds go on
 * until the rest is far enough, and the candidates, one per lane, are put in order by their values in binary64.
 * Logits that are compared themselves have no error but the cut bits.  The groups are looked at in the same way.
 * (All values in binary64 and lists searched anew for every choice: 57 us for 8192 tokens, 8 of 256 experts in 8 groups
 * with a bias; so 10.8 to 14.4 us by the inputs, whose instructions differ by less than 0.1 %: the same ones repeat to 0.1 us.)
 *
 * Bound by instructions, 933 per token of that shape (317 of them the groups', 21 a choice, 39 the exact division of the
 * weights), issued in 62 % of the cycles with 26 warps per SM.  Without groups and bias, 524: 6.7 us.  One token takes a
 * launch, 2.6 to 3 us.
 */
template <int DT, int NI, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(32 * kRouteWarps, NI <= 8 ? 8 : NI <= 16 ? 5 : 3) k_route(const __grid_constant__ RouteArgs a)
{
    __shared__ float s_l[kRouteWarps][NI * 32];
    __shared__ __align__(16) double s_v[kRouteWarps][NI * 32];
    constexpr uint32_t kCut = NI - 1;
    grid_let_next_in();
    const int lane = threadIdx.x & 31;
    const unsigned long long token = (unsigned long long)blockIdx.x * kRouteWarps + threadIdx.x / 32;
    grid_wait();
    if (token >= a.tokens) return;
    float v[NI], *const sl = s_l[threadIdx.x / 32];
    double *const sv = s_v[threadIdx.x / 32];
    load_logits<DT, NI>(v, a.logits, a.P, token * a.ld_logits, a.experts);
    bool nan = false;
#pragma unroll
    for (int j = 0; j < NI; ++j) { sl[j * 32 + lane] = v[j]; nan = nan || v[j] != v[j]; }
    nan = __any_sync(0xFFFFFFFFu, nan);
    if (nan) {                                            /* in the choice: the lowest */
#pragma unroll
        for (int j = 0; j < NI; ++j) if (v[j] != v[j]) v[j] = -INFINITY;
    }

    const bool scored = BIAS || (GROUPS && a.group_score == SIFAR_GROUP_TOP2), softmax = a.score == SIFAR_SCORE_SOFTMAX;
    float top = -INFINITY, sum = 1.0f;                    /* of the softmax over all experts */
    if (softmax && (!a.renormalize || scored)) {
#pragma unroll
        for (int j = 0; j < NI; ++j) top = fmaxf(top, v[j]);
        top = nan ? NAN : of_key(__reduce_max_sync(0xFFFFFFFFu, key_of(top)));
        if (top != -INFINITY) {
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < NI; ++j) sum += expf(v[j] - top);
            sum = sifar::warp_sum(sum);
        }
    }

    /* what is compared, and its error: `fixed`, and `relative` times its size, both for a pair */
    float fixed = 0.0f, relative = 0.0f;
    bool lost = false;                                    /* binary32 does not have the values */
    if (scored) {
        if (softmax) {
            /* l - top, two exponentials, the sum's NI + 5 adds, the division: of a score of at most 1 / sum */
            const float inv = top == -INFINITY ? 0.0f : 1.0f / sum;
            fixed = 2.5f * ((NI + 16) * 0x1p-24f + 0x1p-21f) * inv;
#pragma unroll
            for (int j = 0; j < NI; ++j) v[j] = top == -INFINITY ? 0.0f : __expf(v[j] - top) * inv;
        } else {
            /* 1 / (1 + exp(-l)): the exponential's two steps and its argument's product count s (1 - s) times, the sum and
               the reciprocal s times: below 2^-22 together */
            fixed = 2.5f * 0x1p-22f;
#pragma unroll
            for (int j = 0; j < NI; ++j) v[j] = reciprocal(1.0f + __expf(-v[j]));
        }
        relative = 2.5f * 0x1p-24f + 1.25f * NI * 0x1p-23f;
        if (BIAS) {
#pragma unroll
            for (int j = 0; j < NI; ++j)
                if (is_expert<NI>(j, a.experts)) v[j] += a.bias[j * 32 + lane];
        }
        bool odd = nan;
#pragma unroll
        for (int j = 0; j < NI; ++j) odd = odd || v[j] != v[j];
        lost = __any_sync(0xFFFFFFFFu, odd);
    }
    double total = 1.0;
    bool have_total = !softmax || !scored;
    uint32_t open = 0xFFFFFFFFu;
    if (GROUPS) {
        float *const sf = reinterpret_cast<float *>(sv);
#pragma unroll
        for (int j = 0; j < NI; ++j) sf[j * 32 + lane] = v[j];
        __syncwarp();
        const int shift = group_shift(a.groups), mygroup = lane >> shift;
        const float mine = group_value(sf, a.per, a.groups, shift, a.group_score == SIFAR_GROUP_TOP2);
        uint32_t k = mygroup < a.groups ? key_of(mine) : 0u, least = 0u;
        open = 0u;
        for (int i = 0; i < a.top_groups; ++i) {
            least = __reduce_max_sync(0xFFFFFFFFu, k);
            const int g = (__ffs(__ballot_sync(0xFFFFFFFFu, k == least)) - 1) >> shift;
            open |= 1u << g;
            if (mygroup == g) k = 0u;
        }
        if (scored) {
            const float x = of_key(least), y = of_key(__reduce_max_sync(0xFFFFFFFFu, k));
            /* a sum of two: twice the error, and its own rounding */
            if (lost || !(x - y > 2.0f * fixed + 2.0f * relative * fmaxf(fabsf(x), fabsf(y)))) {
                if (!have_total) total = softmax_total(a, sl, top);
                have_total = true;
                open = groups_exactly(a, sl, sv, top, total);
            }
            if (!BIAS) {
#pragma unroll
                for (int j = 0; j < NI; ++j) v[j] = sl[j * 32 + lane];
                if (nan) {
#pragma unroll
                    for (int j = 0; j < NI; ++j) if (v[j] != v[j]) v[j] = -INFINITY;
                }
            }
        }
    }
    if (!BIAS) { fixed = relative = 0.0f; lost = false; }

    uint32_t in = 0xFFFFFFFFu;                            /* bit j: item j is in an open group */
    if (GROUPS) {
        in = 0u;
        if ((a.per & 31) == 0) {                          /* a group is a.per / 32 items of every lane */
            const int items = a.per >> 5;
            for (uint32_t rest = open; rest; rest &= rest - 1u) in |= ((1u << items) - 1u) << ((__ffs(rest) - 1) * items);
        } else {
#pragma unroll
            for (int j = 0; j < NI; ++j) in |= (open >> ((uint32_t)(j * 32 + lane) * a.per_magic >> 20) & 1u) << j;
        }
    }
    uint32_t key[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const uint32_t u = __float_as_uint(v[j] + 0.0f);
        key[j] = ((u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) & ~kCut) | (kCut - (uint32_t)j);
        if (!is_expert<NI>(j, a.experts) || (GROUPS && !(in >> j & 1u))) key[j] = 0u;
    }
    sort_keys(key);

    uint32_t mykey = 0u;                                  /* lane i: the i-th candidate */
    int owner = 0;
    auto take = [&](int i) {
        const uint32_t k = __reduce_max_sync(0xFFFFFFFFu, key[0]);
        const int who = __ffs(__ballot_sync(0xFFFFFFFFu, key[0] == k)) - 1;
        if (lane == i) { mykey = k; owner = who; }
        const bool pop = lane == who;
#pragma unroll
        for (int j = 0; j + 1 < NI; ++j) key[j] = pop ? key[j + 1] : key[j];
        if (pop) key[NI - 1] = 0u;
        return k;
    };
    auto apart = [&](float x, float y) { return x - y > fixed + relative * fmaxf(fabsf(x), fabsf(y)); };
    for (int i = 0; i < a.top_k; ++i) take(i);
    __syncwarp();
    const bool mine = lane < a.top_k;
    int chosen = (int)(kCut - (mykey & kCut)) * 32 + owner;
    float logit = mine ? sl[chosen] : 0.0f;

    const int last = a.top_k - 1;
    const float x = of_key(mykey & ~kCut), lx = __shfl_sync(0xFFFFFFFFu, x, last);
    const float b = BIAS && mine ? a.bias[chosen] : 0.0f;
    const float nx = __shfl_down_sync(0xFFFFFFFFu, x, 1), nl = __shfl_down_sync(0xFFFFFFFFu, logit, 1);
    const float nb = __shfl_down_sync(0xFFFFFFFFu, b, 1);
    const uint32_t rest = __reduce_max_sync(0xFFFFFFFFu, key[0]);
    const bool sure = lane > last || (lane == last ? rest == 0u || apart(lx, of_key(rest & ~kCut))
                                                   : apart(x, nx) || (logit == nl && b == nb));
    if (lost || !__all_sync(0xFFFFFFFFu, sure)) {
        if (!have_total) total = softmax_total(a, sl, top);
        /* candidates: as many more as are not far from the last one */
        int n = a.top_k;
        for (uint32_t k = __reduce_max_sync(0xFFFFFFFFu, key[0]);
             k != 0u && n < 32 && !lost && !apart(lx, of_key(k & ~kCut)); k = __reduce_max_sync(0xFFFFFFFFu, key[0]))
            take(n++);
        const uint32_t k = __reduce_max_sync(0xFFFFFFFFu, key[0]);
        if (lost || !(k == 0u || apart(lx, of_key(k & ~kCut)))) {
            chosen = choose_exactly<NI>(a, sl, sv, top, total, open);
        } else {
            const int e = (int)(kCut - (mykey & kCut)) * 32 + owner;
            chosen = order_exactly(a, sl, reinterpret_cast<int *>(sv), top, total, e, n);
        }
        logit = mine ? sl[chosen] : 0.0f;
    }

    float w;
    if (a.renormalize) {
        float max = of_key(__reduce_max_sync(0xFFFFFFFFu, mine ? key_of(logit) : 0u));
        if (nan && __any_sync(0xFFFFFFFFu, mine && logit != logit)) max = NAN;
        w = softmax ? expf(logit - max) : scaled_sigmoid(logit, max);
        if (!mine || max == -INFINITY) w = 0.0f;
        const float total = sifar::warp_sum(w);
        w = max == -INFINITY ? 0.0f : w / total;
    } else if (softmax) {
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
__global__ void __launch_bounds__(32 * kRouteWarps) k_route_grad(const __grid_constant__ RouteGradArgs a)
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

template <int DT, int NI>
static cudaError_t launch_route_n(dim3 grid, cudaStream_t stream, const RouteArgs &a)
{
    const dim3 block(32 * kRouteWarps);
    if (a.bias)
        return a.groups > 1 ? launch_op(k_route<DT, NI, true, true>, grid, block, 1, 0, stream, a)
                            : launch_op(k_route<DT, NI, true, false>, grid, block, 1, 0, stream, a);
    return a.groups > 1 ? launch_op(k_route<DT, NI, false, true>, grid, block, 1, 0, stream, a)
                        : launch_op(k_route<DT, NI, false, false>, grid, block, 1, 0, stream, a);
}

template <int DT>
static cudaError_t launch_route(dim3 grid, cudaStream_t stream, const RouteArgs &a)
{
    if (a.experts <= 64) return launch_route_n<DT, 2>(grid, stream, a);
    if (a.experts <= 128) return launch_route_n<DT, 4>(grid, stream, a);
    if (a.experts <= 256) return launch_route_n<DT, 8>(grid, stream, a);
    if (a.experts <= 512) return launch_route_n<DT, 16>(grid, stream, a);
    return launch_route_n<DT, 32>(grid, stream, a);
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
    a.per = a.experts / a.groups;
    a.per_magic = ((1u << 20) + (uint32_t)a.per - 1u) / (uint32_t)a.per;
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
