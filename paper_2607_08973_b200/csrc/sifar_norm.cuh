/*
 * How the norm kernels lay a row over threads, and the sums over a row.
 *
 * A thread holds 16, 32 or 64 bytes of every array of a row in registers from its first load to its last store, so a row
 * is read once however many sums go over it.  A row takes `tx` threads of a CTA; where it is longer than a CTA of
 * kMaxRowThreads holds, a cluster of up to eight CTAs has it and its sums meet in their shared memory.
 */
#ifndef SIFAR_NORM_CUH
#define SIFAR_NORM_CUH

#include <atomic>

#include "sifar_norm_shape.cuh"
#include "sifar_ops.cuh"

namespace sifar {

/*
 * How a kernel reaches its rows.
 *   kWhole    every row of every array starts on a 16-byte boundary: a vector is one access.
 *   kShifted  rows start anywhere, as contiguous rows of an odd number of columns do: a vector is put together from the two
 *             aligned ones that it lies in, and stored in the largest pieces that its address allows.
 *             (4096 x 4097 bf16 of one rank: 53 us forward and 142 back, by elements 77 and 244.)
 *   kElement  single elements, neighbours by neighbouring threads.
 */
enum Access { kWhole, kShifted, kElement };

/* The form of a kernel: element type, 32-bit words of a row and array per thread, access. */
template <int DT_, int W_, Access A_> struct Form {
    static constexpr int DT = DT_, W = W_;
    static constexpr Access ACCESS = A_;
    static constexpr bool VEC = A_ != kElement;
    using T = typename Elem<DT_>::type;
    static constexpr uint32_t es = sizeof(T);
    static constexpr int items = W_ * 4 / (int)sizeof(T), pairs = items / 2;
    static constexpr int vectors = W_ / 4, vector_pairs = pairs / vectors;       /* of 16 bytes */
    static_assert(A_ != kShifted || DT_ == SIFAR_BF16, "fp32 elements are words: single ones do");
    static_assert(SIFAR_NORM_MAX_COLS <= items * kMaxRowThreads * (int)kMaxNormCluster, "columns that a cluster holds");
};

/* The columns of a thread: item j is column at(j).  VEC: runs of 16 bytes, else single elements. */
template <typename F> struct Columns {
    static constexpr int N = F::items;
    static constexpr int EPV = F::VEC ? Elem<F::DT>::per_vec : 1;      /* neighbours that are fetched together */
    uint32_t first, step, cols;
    __device__ __forceinline__ Columns(uint32_t part, uint32_t tx, uint32_t t, uint32_t cols_)
        : first(part * N * tx + t * EPV), step(tx * EPV), cols(cols_) {}
    __device__ __forceinline__ uint32_t at(int j) const { return first + (uint32_t)(j / EPV) * step + (uint32_t)(j % EPV); }
    __device__ __forceinline__ bool has(int j) const { return at(j) < cols; }
};

/*
 * The thread's 16-byte vectors of a row: byte offsets (0 where the row has ended, so that a load may go there all the
 * same and its value is left out later), which of them exist, and whether the warp holds the row's last, short vector
 * (ragged) and looks at every element.  Computed once: all rows are alike.
 */
template <typename F> struct Lane {
    uint32_t at[F::vectors];
    bool in[F::vectors];
    bool ragged;
    __device__ __forceinline__ explicit Lane(const Columns<F> &c)
    {
        bool cut = !F::VEC || c.cols == 0;                /* a row that is not there: nothing is read */
#pragma unroll
        for (int v = 0; v < F::vectors; ++v) {
            const uint32_t i = c.at(v * c.EPV);
            in[v] = i < c.cols;
            at[v] = in[v] ? i * F::es : 0u;
            cut = cut || (in[v] && i + c.EPV > c.cols);
        }
        ragged = __any_sync(0xFFFFFFFFu, cut);
    }
};

/* The thread's items of one row as they lie in memory. */
template <typename F> struct Raw { uint32_t w[F::W]; };

/* Four words (vector v), every element looked at: absent ones are 0. */
template <typename F>
__device__ __forceinline__ void load_each(Raw<F> &x, int v, const void *row, const Columns<F> &c)
{
    using T = typename F::T;
    const T *p = static_cast<const T *>(row);
#pragma unroll
    for (int i = 4 * v; i < 4 * v + 4; ++i) {
        if (F::DT == SIFAR_F32) {
            x.w[i] = c.has(i) ? (uint32_t)p[c.at(i)] : 0u;
        } else {
            const uint32_t lo = c.has(2 * i) ? (uint32_t)p[c.at(2 * i)] : 0u, hi = c.has(2 * i + 1) ? (uint32_t)p[c.at(2 * i + 1)] : 0u;
            x.w[i] = lo | hi << 16;
        }
    }
}

/* An aligned vector; where the row has ended, some other element of it (or of the next row, behind a short vector). */
template <typename F>
__device__ __forceinline__ void load_whole(Raw<F> &x, int v, const void *row, const Lane<F> &l)
{
    const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const char *>(row) + l.at[v]);
    x.w[4 * v] = q.x;
    x.w[4 * v + 1] = q.y;
    x.w[4 * v + 2] = q.z;
    x.w[4 * v + 3] = q.w;
}

/* Vector v that starts m bytes into two aligned ones: their eight words moved down. */
template <typename F> __device__ __forceinline__ void shift_vectors(Raw<F> &x, int v, const uint4 &a, const uint4 &b, uint32_t m)
{
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = m & 8u ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = m & 4u ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) x.w[4 * v + i] = __funnelshift_r(w[i], w[i + 1], (m & 2u) * 8u);
}
template <typename F>
__device__ __forceinline__ void load_shifted(Raw<F> &x, int v, const void *row, const Lane<F> &l)
{
    const uintptr_t p = (uintptr_t)row + l.at[v];
    const uint32_t m = (uint32_t)p & 15u;
    const uint4 *g = reinterpret_cast<const uint4 *>(p - m);
    shift_vectors(x, v, g[0], g[m ? 1 : 0], m);
}

/* Whether the warp looks at every element of the row: at its ragged end (vectors of which the items behind it are cut
   off again were slower: 33 us against 28 for 1003 x 4099 fp32), and in the array's first and last row (`edge`) where a
   shifted vector might reach out of the array.  The caller branches on it once and passes the constant. */
template <typename F> __device__ __forceinline__ bool by_element(const Lane<F> &l, bool edge)
{
    return F::ACCESS == kElement || l.ragged || (F::ACCESS == kShifted && edge);
}
template <typename F>
__device__ __forceinline__ void load_vector(Raw<F> &x, int v, const void *row, const Columns<F> &c, const Lane<F> &l, bool each)
{
    if (F::ACCESS == kElement || each) load_each(x, v, row, c);
    else if constexpr (F::ACCESS == kShifted) load_shifted(x, v, row, l);
    else load_whole(x, v, row, l);
}
template <typename F>
__device__ __forceinline__ void load_row(Raw<F> &x, const void *row, const Columns<F> &c, const Lane<F> &l, bool each)
{
#pragma unroll
    for (int v = 0; v < F::vectors; ++v) load_vector(x, v, row, c, l, each);
}

/* Weights and gate rows, whatever the alignment of the rows: nothing around them is read. */
template <typename F>
__device__ __forceinline__ void load_weight(Raw<F> &x, const void *row, const Columns<F> &c, const Lane<F> &l)
{
    const bool whole = F::VEC && !l.ragged && ((uintptr_t)row & 15u) == 0;
#pragma unroll
    for (int v = 0; v < F::vectors; ++v) {
        if (whole) load_whole(x, v, row, l);
        else load_each(x, v, row, c);
    }
}

/*
 * A thread's items in binary32, two by two: the arithmetic takes two per instruction (the packed forms round each half
 * as the plain ones do).
 */
template <typename F> struct Items {
    static constexpr int N = F::pairs;
    float2 p[N];
};
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

template <typename F> __device__ __forceinline__ float2 pair(const Raw<F> &x, int i)
{
    if (F::DT == SIFAR_BF16) return make_float2(bf16lo_to_f32(x.w[i % F::W]), bf16hi_to_f32(x.w[i % F::W]));
    return make_float2(__uint_as_float(x.w[(2 * i) % F::W]), __uint_as_float(x.w[(2 * i + 1) % F::W]));
}
template <typename F> __device__ __forceinline__ Items<F> items(const Raw<F> &x)
{
    Items<F> f;
#pragma unroll
    for (int i = 0; i < f.N; ++i) f.p[i] = pair<F>(x, i);
    return f;
}
template <typename F> __device__ __forceinline__ Items<F> all_items(float v)
{
    Items<F> f;
#pragma unroll
    for (int i = 0; i < f.N; ++i) f.p[i] = both(v);
    return f;
}

/* acc += items of x, one binary32 add each */
template <typename F> __device__ __forceinline__ void add_pair(float2 &acc, const Raw<F> &x, int i)
{
    if (F::DT == SIFAR_BF16) acc = make_float2(add_bf16lo(acc.x, x.w[i % F::W]), add_bf16hi(acc.y, x.w[i % F::W]));
    else acc = __fadd2_rn(acc, pair<F>(x, i));
}
template <typename F> __device__ __forceinline__ void add_items(Items<F> &acc, const Raw<F> &x)
{
#pragma unroll
    for (int i = 0; i < acc.N; ++i) add_pair<F>(acc.p[i], x, i);
}

/* weight + offset, or 1 where there is no weight.  A vector behind the row's end, in whose place load_whole reads the row's
   first, is 0: an infinite weight times the zeros there would make the row's sums NaN. */
template <typename F>
__device__ __forceinline__ Items<F> load_factor(const void *weight, float offset, const Columns<F> &c, const Lane<F> &l)
{
    if (!weight) return all_items<F>(1.0f);
    Raw<F> w;
    load_weight(w, weight, c, l);
    Items<F> f = items<F>(w);
#pragma unroll
    for (int i = 0; i < f.N; ++i) f.p[i] = F::VEC && !l.in[i / F::vector_pairs] ? both(0.0f) : __fadd2_rn(f.p[i], both(offset));
    return f;
}

template <typename F>
__device__ __forceinline__ void store_items(void *row, const Items<F> &f, const Columns<F> &c, const Lane<F> &l)
{
    using T = typename F::T;
#pragma unroll
    for (int v = 0; v < F::vectors; ++v) {
        constexpr int N = F::vector_pairs;                /* 4 of bf16, 2 of fp32 */
        const float2 *p = &f.p[v * N];
        if (F::ACCESS == kElement || (l.ragged && c.at(v * c.EPV) + c.EPV > c.cols)) {
#pragma unroll
            for (int j = 2 * N * v; j < 2 * N * (v + 1); ++j)
                if (c.has(j)) static_cast<T *>(row)[c.at(j)] = narrow<F::DT>((j & 1) ? f.p[j / 2].y : f.p[j / 2].x);
            continue;
        }
        if (!l.in[v]) continue;
        uint4 q;
        if (F::DT == SIFAR_BF16)
            q = make_uint4(f32x2_to_bf16x2(p[0].x, p[0].y), f32x2_to_bf16x2(p[1].x, p[1].y), f32x2_to_bf16x2(p[2 % N].x, p[2 % N].y),
                           f32x2_to_bf16x2(p[3 % N].x, p[3 % N].y));
        else
            q = make_uint4(__float_as_uint(p[0].x), __float_as_uint(p[0].y), __float_as_uint(p[1].x), __float_as_uint(p[1].y));
        char *const to = static_cast<char *>(row) + l.at[v];
        const uint32_t m = F::ACCESS == kWhole ? 0u : (uint32_t)(uintptr_t)to & 15u;
        if (m == 0u) {
            *reinterpret_cast<uint4 *>(to) = q;
        } else if ((m & 7u) == 0u) {
            reinterpret_cast<uint2 *>(to)[0] = make_uint2(q.x, q.y);
            reinterpret_cast<uint2 *>(to)[1] = make_uint2(q.z, q.w);
        } else if ((m & 3u) == 0u) {
            uint32_t *const w = reinterpret_cast<uint32_t *>(to);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else {                                          /* bf16 at an odd element: half a word, three words, half a word */
            *reinterpret_cast<uint16_t *>(to) = (uint16_t)q.x;
            uint32_t *const w = reinterpret_cast<uint32_t *>(to + 2);
            w[0] = __funnelshift_r(q.x, q.y, 16);
            w[1] = __funnelshift_r(q.y, q.z, 16);
            w[2] = __funnelshift_r(q.z, q.w, 16);
            *reinterpret_cast<uint16_t *>(to + 14) = (uint16_t)(q.w >> 16);
        }
    }
}

/* Sum of the squares of the items that exist. */
template <typename F>
__device__ __forceinline__ float squares(const Items<F> &f, const Lane<F> &l)
{
    constexpr int N = F::vector_pairs;
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < F::vectors; ++v) {
        float2 q = __fmul2_rn(f.p[v * N], f.p[v * N]);
#pragma unroll
        for (int i = 1; i < N; ++i) q = __ffma2_rn(f.p[v * N + i], f.p[v * N + i], q);
        sum += F::VEC && !l.in[v] ? 0.0f : q.x + q.y;
    }
    return sum;
}

/* Items to a binary32 array (sums over rows). */
template <typename F>
__device__ __forceinline__ void store_f32(float *row, const Items<F> &f, const Columns<F> &c)
{
    const bool wide = F::VEC && ((uintptr_t)row & 15u) == 0;
#pragma unroll
    for (int j = 0; j < F::items; j += 4) {
        const float4 q = make_float4(f.p[j / 2].x, f.p[j / 2].y, f.p[j / 2 + 1].x, f.p[j / 2 + 1].y);
        if (wide && c.at(j) + 4 <= c.cols) {
            *reinterpret_cast<float4 *>(row + c.at(j)) = q;
        } else {
            if (c.has(j)) row[c.at(j)] = q.x;
            if (c.has(j + 1)) row[c.at(j + 1)] = q.y;
            if (c.has(j + 2)) row[c.at(j + 2)] = q.z;
            if (c.has(j + 3)) row[c.at(j + 3)] = q.w;
        }
    }
}

/*
 * Sums of N values over the threads of one row: warps by shuffles, a CTA's warps in order through shared memory, a
 * cluster's CTAs in rank order through its distributed shared memory.  All threads of the CTA (cluster) call it
 * together; calls use two places in turn, so that a fast warp or CTA does not overwrite what a slow one still reads
 * (whoever has come to the call after next has seen that all have passed the next one's barrier).
 * Between CTAs each value travels with the call's number in one word, which the readers poll for: a cluster barrier
 * would wait for the rows' stores as well (1003 x 4099 fp32, three ranks: 52 us with barriers, 42 with words).  CTAs of a
 * cluster run at the same time, so the wait ends; its limit is there for the case that it does not: the sum is NaN then.
 */
template <int N> struct RowSum {
    float4 warps[2][N][kMaxRowThreads / 32]; /* [turn][value][row of the CTA * vectors per row]: a word per warp, 0 behind the last */
    unsigned long long parts[2][N][kMaxNormCluster];
};
constexpr int kPartPolls = 1 << 22;
__host__ __device__ inline uint32_t sum_vectors(uint32_t tx) { return (tx / 32 + 3) / 4; }

/* Before the first sum; a barrier (of the cluster) must follow. */
template <int N> __device__ __forceinline__ void clear_row_sum(RowSum<N> &s)
{
    static_assert(sizeof(RowSum<N>) % 16 == 0, "cleared by vectors");
    for (uint32_t i = threadIdx.y * blockDim.x + threadIdx.x; i < sizeof s / 16; i += blockDim.x * blockDim.y)
        reinterpret_cast<float4 *>(&s)[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}

/* Sums of three values over a warp with six exchanges: halves of the warp take over different values, then quarters.
   Every lane of quarter k has the total of value k (k = 3: 0). */
__device__ __forceinline__ float warp_sum3(float a, float b, float c)
{
    const uint32_t lane = threadIdx.x & 31u;
    const bool up = lane & 16u, odd = lane & 8u;
    float x = (up ? c : a) + __shfl_xor_sync(0xFFFFFFFFu, up ? a : c, 16);          /* a below, c above */
    float y = (up ? 0.0f : b) + __shfl_xor_sync(0xFFFFFFFFu, up ? b : 0.0f, 16);    /* b below, 0 above */
    x = (odd ? y : x) + __shfl_xor_sync(0xFFFFFFFFu, odd ? x : y, 8);               /* a, b, c, 0 */
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

struct RowPlace {
    uint32_t tx, t, row, parts, part;        /* threads of a row, which of them, row of the CTA, CTAs of a row, which of them */
};

/*
 * A sum in three steps, so that other work can lie between: publish_sums (a barrier of the CTA must follow, where a row
 * has more than a warp), send_sums (clusters), collect_sums.  `call` counts the sums from 0.
 */
template <int N> __device__ __forceinline__ void publish_sums(float (&v)[N], RowSum<N> &s, uint32_t call, const RowPlace &p)
{
    static_assert(N == 1 || N == 3, "one value or three");
    float x;
    if (N == 1) x = warp_sum(v[0]);
    else x = warp_sum3(v[0], v[1 % N], v[2 % N]);         /* lane 8 k: value k */
    if (p.tx > 32) {
        const uint32_t lane = p.t & 31u;
        if (N == 1 ? lane == 0 : (lane & 7u) == 0 && lane < 24u)
            reinterpret_cast<float *>(&s.warps[call & 1u][lane / 8][p.row * sum_vectors(p.tx)])[p.t / 32] = x;
    } else if (N == 1) {
        v[0] = x;
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xFFFFFFFFu, x, 8 * k);
    }
}

/* The CTA's own totals.  Three values: every lane adds four warps' parts of one of them, the lanes of a value meet by
   exchanges; twelve vectors read and added by every thread would be 50 instructions for 12.  All lanes of a warp call. */
template <int N> __device__ __forceinline__ void local_sums(float (&v)[N], const RowSum<N> &s, uint32_t call, const RowPlace &p)
{
    constexpr uint32_t kVectors = kMaxRowThreads / 128;      /* of a value at most */
    const uint32_t n = sum_vectors(p.tx), lane = p.t & 31u;
    if (N == 1) {
        const float4 *w = &s.warps[call & 1u][0][p.row * n];
        float2 x = make_float2(0.0f, 0.0f);
#pragma unroll
        for (uint32_t i = 0; i < kVectors; ++i)
            if (i < n) { const float4 q = w[i]; x = __fadd2_rn(x, __fadd2_rn(make_float2(q.x, q.y), make_float2(q.z, q.w))); }
        v[0] = x.x + x.y;
        return;
    }
    static_assert(kVectors == 4, "lane 4 k + i: vector i of value k");
    float x = 0.0f;
    if ((lane & 3u) < n && lane < 4 * N) {
        const float4 q = s.warps[call & 1u][lane / 4 % N][p.row * n + (lane & 3u)];
        x = (q.x + q.y) + (q.z + q.w);
    }
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xFFFFFFFFu, x, 4 * k);
}

template <int N> __device__ __forceinline__ void send_sums(RowSum<N> &s, uint32_t call, const RowPlace &p)
{
    if (p.t < 32u) {
        float v[N];
        local_sums(v, s, call, p);
        if (p.t < p.parts) {
#pragma unroll
            for (int k = 0; k < N; ++k) store_cluster_tagged(&s.parts[call & 1u][k][p.part], p.t, v[k], call + 1u);
        }
    }
}

/* In: what publish_sums left.  Out: the row's totals. */
template <int N> __device__ __forceinline__ void collect_sums(float (&v)[N], const RowSum<N> &s, uint32_t call, const RowPlace &p)
{
    if (p.parts == 1) {
        if (p.tx > 32) local_sums(v, s, call, p);
        return;
    }
    int polls = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float x = 0.0f;
        for (uint32_t i = 0; i < p.parts; ++i) {
            unsigned long long w = load_tagged(&s.parts[call & 1u][k][i]);
            while ((uint32_t)(w >> 32) != call + 1u && ++polls < kPartPolls) w = load_tagged(&s.parts[call & 1u][k][i]);
            x += (uint32_t)(w >> 32) == call + 1u ? __uint_as_float((uint32_t)w) : NAN;
        }
        v[k] = x;
    }
}

/* The three in a row. */
template <int N> __device__ __forceinline__ void row_sums(float (&v)[N], RowSum<N> &s, uint32_t call, const RowPlace &p)
{
    publish_sums(v, s, call, p);
    if (p.tx > 32) __syncthreads();
    if (p.parts > 1) send_sums(s, call, p);
    collect_sums(v, s, call, p);
}

/* 1 / sqrt(mean + eps) */
__device__ __forceinline__ float rrms(float sum, uint32_t cols, float eps) { return rsqrtf(sum / (float)cols + eps); }

/*
 * Rows that are under way while others are worked on: a ring of shared memory that each thread fills with its own items
 * by asynchronous copies and reads itself, so that no barrier goes with it.  A place (an array of a row) holds the
 * threads' words side by side, 16 bytes each (VEC) or 4.
 */
template <typename F> struct Ring {
    static_assert(F::ACCESS != kElement || F::DT == SIFAR_F32, "a copy moves 4 bytes at least");
    static constexpr bool shifted = F::ACCESS == kShifted;
    static constexpr uint32_t unit = F::VEC ? 16 : 4;
    static constexpr int copies = shifted ? 2 : 1;                   /* of a vector: the two aligned ones around it */
    static constexpr uint32_t bytes = sizeof(Raw<F>) * copies;       /* per thread and array */
    static constexpr int N = sizeof(Raw<F>) / unit;
    uint32_t first, threads;                                         /* the thread's place in slot 0; of the CTA */
    uint32_t from[N], n[N];                                          /* of each unit: bytes into the row, bytes to move (the rest becomes 0) */
    uint32_t row_bytes;
    __device__ __forceinline__ Ring(const void *smem, const Columns<F> &c)
    {
        threads = blockDim.x * blockDim.y;
        first = (uint32_t)__cvta_generic_to_shared(smem) + (threadIdx.y * blockDim.x + threadIdx.x) * unit;
        row_bytes = c.cols * F::es;
#pragma unroll
        for (int v = 0; v < N; ++v) {
            const uint32_t i = c.at(v * c.EPV);
            n[v] = i < c.cols ? min((uint32_t)c.EPV, c.cols - i) * F::es : 0u;
            from[v] = n[v] ? i * F::es : 0u;
        }
    }
    __device__ __forceinline__ void copy(uint32_t to, const char *p, uint32_t bytes_) const
    {
        if (F::VEC) asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(p), "r"(bytes_) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(to), "l"(p), "r"(bytes_) : "memory");
    }
    /* a row of an array to place `at` (bytes; a place takes threads * bytes) */
    __device__ __forceinline__ void fetch(uint32_t at, const void *row) const
    {
        const uint32_t to = first + at;
#pragma unroll
        for (int v = 0; v < N; ++v) {
            const char *p = static_cast<const char *>(row) + from[v];
            if (shifted) {
                /* up to the row's end: what follows becomes 0.  The bytes before the row in its first vector are the row
                   before's and are moved out */
                const uint32_t m = (uint32_t)(uintptr_t)p & 15u, end = n[v] ? row_bytes - from[v] + m : 0u;
                copy(to + 2 * v * threads * unit, p - m, min(16u, end));
                copy(to + (2 * v + 1) * threads * unit, end > 16u ? p - m + 16 : p - m, m && end > 16u ? min(16u, end - 16u) : 0u);
            } else if (F::VEC) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to + v * threads * unit), "l"(p), "r"(n[v]) : "memory");
            } else {
                copy(to + v * threads * unit, p, n[v]);
            }
        }
    }
    __device__ __forceinline__ void commit() const { asm volatile("cp.async.commit_group;" ::: "memory"); }
    /* until all but the last k groups of this thread are there */
    __device__ __forceinline__ void wait(uint32_t k) const
    {
        if (k == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
        else if (k == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else if (k == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else asm volatile("cp.async.wait_group 3;" ::: "memory");
    }
    /* words 4 v to 4 v + 3 of the thread; `row`: where the array's row starts.  Plain loads: the compiler puts those of a
       row side by side, but not before the wait or behind the fetch that comes after them */
    __device__ __forceinline__ void read_vector(Raw<F> &x, int v, const unsigned char *smem, uint32_t at, const void *row) const
    {
        const unsigned char *p = smem + at + (threadIdx.y * blockDim.x + threadIdx.x) * unit;
        if constexpr (shifted) {
            shift_vectors(x, v, *reinterpret_cast<const uint4 *>(p + 2 * v * threads * unit),
                          *reinterpret_cast<const uint4 *>(p + (2 * v + 1) * threads * unit), (uint32_t)(uintptr_t)row & 15u);
        } else if (F::VEC) {
            const uint4 q = *reinterpret_cast<const uint4 *>(p + v * threads * unit);
            x.w[4 * v] = q.x;
            x.w[4 * v + 1] = q.y;
            x.w[4 * v + 2] = q.z;
            x.w[4 * v + 3] = q.w;
        } else {
#pragma unroll
            for (int i = 4 * v; i < 4 * v + 4; ++i) x.w[i] = *reinterpret_cast<const uint32_t *>(p + i * threads * unit);
        }
    }
};

}  /* namespace sifar */
#endif
