/*
 * How the norm kernels lay a row over threads, and the sum over a row.
 *
 * A thread holds kItems elements of a row in registers from its first load to its last store, so a row is read once
 * however many sums go over it.  A row takes `tx` threads of a CTA; where it is longer than kMaxRowThreads * kItems
 * elements, a cluster of up to eight CTAs holds it and its sums meet in their shared memory.
 */
#ifndef SIFAR_NORM_CUH
#define SIFAR_NORM_CUH

#include <atomic>

#include "sifar_ops.cuh"

namespace sifar {

constexpr int kItems = 8;                    /* elements of a row per thread: 16 bytes of bf16, 2 x 16 bytes of fp32 */
constexpr int kMaxRowThreads = 512;
constexpr unsigned kMaxNormCluster = 8;
static_assert(SIFAR_NORM_MAX_COLS == kItems * kMaxRowThreads * (int)kMaxNormCluster, "columns a cluster holds");

/* The columns of a thread: item j is column at(j). */
template <int DT, bool VEC> struct Columns {
    static constexpr int EPV = VEC ? Elem<DT>::per_vec : 1;      /* neighbours that are fetched together */
    static constexpr int NV = kItems / EPV;
    uint32_t first, step, cols;
    __device__ __forceinline__ Columns(uint32_t part, uint32_t tx, uint32_t t, uint32_t cols_)
        : first((part * NV * tx + t) * EPV), step(tx * EPV), cols(cols_) {}
    __device__ __forceinline__ uint32_t at(int j) const { return first + (uint32_t)(j / EPV) * step + (uint32_t)(j % EPV); }
    __device__ __forceinline__ bool has(int j) const { return at(j) < cols; }
};

/*
 * The thread's 16-byte vectors of a row: byte offsets (0 where the row has ended, so that a load may go there all the
 * same and its value is left out later), which of them exist, and whether the warp holds the row's last, short vector
 * and has to look at every element.  Computed once: all rows are alike.
 */
template <int DT, bool VEC> struct Lane {
    static constexpr int NV = VEC ? Columns<DT, VEC>::NV : 1;
    uint32_t at[NV];
    bool in[NV];
    bool ragged;
    __device__ __forceinline__ explicit Lane(const Columns<DT, VEC> &c)
    {
        constexpr uint32_t es = sizeof(typename Elem<DT>::type);
        bool cut = !VEC;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const uint32_t i = c.at(v * c.EPV);
            in[v] = i < c.cols;
            at[v] = in[v] ? i * es : 0u;
            cut = cut || (in[v] && i + c.EPV > c.cols);
        }
        ragged = __any_sync(0xFFFFFFFFu, cut);
    }
};

/* The thread's items of one row as they lie in memory: packed words. */
template <int DT> struct Raw { uint32_t w[kItems / (DT == SIFAR_BF16 ? 2 : 1)]; };

template <int DT, bool VEC>
__device__ __forceinline__ void load_row(Raw<DT> &x, const void *row, const Columns<DT, VEC> &c)
{
    using T = typename Elem<DT>::type;
    const T *p = static_cast<const T *>(row);
    constexpr int W = VEC ? 4 : 1;
    if (VEC) {
#pragma unroll
        for (int v = 0; v < Columns<DT, VEC>::NV; ++v) {
            const uint32_t i = c.at(v * c.EPV);
            uint4 q = make_uint4(0u, 0u, 0u, 0u);
            if (i + c.EPV <= c.cols) {
                q = *reinterpret_cast<const uint4 *>(p + i);
            } else if (i < c.cols) {                      /* the row's last, short vector */
                uint32_t t[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int k = 0; k < c.EPV; ++k)
                    if (i + k < c.cols) {
                        if (DT == SIFAR_BF16) t[k / 2] |= (uint32_t)p[i + k] << (16 * (k & 1));
                        else t[k & 3] = p[i + k];
                    }
                q = make_uint4(t[0], t[1], t[2], t[3]);
            }
            x.w[(v * W + 0) % (sizeof x.w / 4)] = q.x;
            x.w[(v * W + 1) % (sizeof x.w / 4)] = q.y;
            x.w[(v * W + 2) % (sizeof x.w / 4)] = q.z;
            x.w[(v * W + 3) % (sizeof x.w / 4)] = q.w;
        }
    } else if (DT == SIFAR_BF16) {
#pragma unroll
        for (int j = 0; j < kItems; j += 2) {
            const uint32_t lo = c.has(j) ? (uint32_t)p[c.at(j)] : 0u, hi = c.has(j + 1) ? (uint32_t)p[c.at(j + 1)] : 0u;
            x.w[(j / 2) % (sizeof x.w / 4)] = lo | hi << 16;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kItems; ++j) x.w[j % (sizeof x.w / 4)] = c.has(j) ? (uint32_t)p[c.at(j)] : 0u;
    }
}

/* The same where the array may lack the rows' alignment (weights, gates). */
template <int DT, bool VEC>
__device__ __forceinline__ void load_any(Raw<DT> &x, const void *row, const Columns<DT, VEC> &c)
{
    if (!VEC || ((uintptr_t)row & 15u) == 0) { load_row(x, row, c); return; }
    using T = typename Elem<DT>::type;
    const T *p = static_cast<const T *>(row);
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const uint32_t q = c.has(j) ? (uint32_t)p[c.at(j)] : 0u;
        if (DT == SIFAR_F32) x.w[j % (sizeof x.w / 4)] = q;
        else x.w[j / 2 % (sizeof x.w / 4)] = (j & 1) ? x.w[j / 2 % (sizeof x.w / 4)] | q << 16 : q;
    }
}

/*
 * A thread's items in binary32, two by two: the arithmetic below takes two per instruction (the packed forms round
 * each half as the plain ones do).
 */
struct Items {
    float2 p[kItems / 2];
};
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

/* Whole vectors of a row (its warp is not ragged); what lies behind the row's end is some other element of it. */
template <int DT, bool VEC>
__device__ __forceinline__ void load_whole(Raw<DT> &x, const void *row, const Lane<DT, VEC> &l)
{
#pragma unroll
    for (int v = 0; v < Lane<DT, VEC>::NV; ++v) {
        const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const char *>(row) + l.at[v]);
        x.w[(4 * v) % (sizeof x.w / 4)] = q.x;
        x.w[(4 * v + 1) % (sizeof x.w / 4)] = q.y;
        x.w[(4 * v + 2) % (sizeof x.w / 4)] = q.z;
        x.w[(4 * v + 3) % (sizeof x.w / 4)] = q.w;
    }
}

template <int DT> __device__ __forceinline__ float2 pair(const Raw<DT> &x, int i)
{
    if (DT == SIFAR_BF16) return make_float2(bf16lo_to_f32(x.w[i]), bf16hi_to_f32(x.w[i]));
    return make_float2(__uint_as_float(x.w[(2 * i) % (sizeof x.w / 4)]), __uint_as_float(x.w[(2 * i + 1) % (sizeof x.w / 4)]));
}
template <int DT> __device__ __forceinline__ Items items(const Raw<DT> &x)
{
    Items f;
#pragma unroll
    for (int i = 0; i < kItems / 2; ++i) f.p[i] = pair(x, i);
    return f;
}
__device__ __forceinline__ Items all_items(float v)
{
    Items f;
#pragma unroll
    for (int i = 0; i < kItems / 2; ++i) f.p[i] = both(v);
    return f;
}

/* acc += the items of x, one binary32 add each */
template <int DT> __device__ __forceinline__ void add_items(Items &acc, const Raw<DT> &x)
{
#pragma unroll
    for (int i = 0; i < kItems / 2; ++i) {
        if (DT == SIFAR_BF16) acc.p[i] = make_float2(add_bf16lo(acc.p[i].x, x.w[i]), add_bf16hi(acc.p[i].y, x.w[i]));
        else acc.p[i] = __fadd2_rn(acc.p[i], pair(x, i));
    }
}

/* weight + offset, or 1 where there is no weight */
template <int DT, bool VEC>
__device__ __forceinline__ Items load_factor(const void *weight, float offset, const Columns<DT, VEC> &c)
{
    if (!weight) return all_items(1.0f);
    Raw<DT> w;
    load_any(w, weight, c);
    Items f = items(w);
#pragma unroll
    for (int i = 0; i < kItems / 2; ++i) f.p[i] = __fadd2_rn(f.p[i], both(offset));
    return f;
}

template <int DT, bool VEC>
__device__ __forceinline__ void store_row(void *row, const Items &f, const Columns<DT, VEC> &c)
{
    using T = typename Elem<DT>::type;
    T *p = static_cast<T *>(row);
#pragma unroll
    for (int v = 0; v < Columns<DT, VEC>::NV; ++v) {
        const uint32_t i = c.at(v * c.EPV);
        if (VEC && i + c.EPV <= c.cols) {
            uint4 q;
            if (DT == SIFAR_BF16)
                q = make_uint4(f32x2_to_bf16x2(f.p[0].x, f.p[0].y), f32x2_to_bf16x2(f.p[1].x, f.p[1].y),
                               f32x2_to_bf16x2(f.p[2].x, f.p[2].y), f32x2_to_bf16x2(f.p[3].x, f.p[3].y));
            else
                q = make_uint4(__float_as_uint(f.p[(2 * v) % 4].x), __float_as_uint(f.p[(2 * v) % 4].y),
                               __float_as_uint(f.p[(2 * v + 1) % 4].x), __float_as_uint(f.p[(2 * v + 1) % 4].y));
            *reinterpret_cast<uint4 *>(p + i) = q;
        } else {
#pragma unroll
            for (int k = 0; k < c.EPV; ++k) {
                const int j = v * c.EPV + k;
                if (i + k < c.cols) p[i + k] = narrow<DT>((j & 1) ? f.p[j / 2].y : f.p[j / 2].x);
            }
        }
    }
}

template <int DT, bool VEC>
__device__ __forceinline__ void store_items(void *row, const Items &f, const Columns<DT, VEC> &c, const Lane<DT, VEC> &l)
{
    if (l.ragged) { store_row(row, f, c); return; }
#pragma unroll
    for (int v = 0; v < Lane<DT, VEC>::NV; ++v) {
        if (!l.in[v]) continue;
        uint4 q;
        if (DT == SIFAR_BF16)
            q = make_uint4(f32x2_to_bf16x2(f.p[0].x, f.p[0].y), f32x2_to_bf16x2(f.p[1].x, f.p[1].y),
                           f32x2_to_bf16x2(f.p[2].x, f.p[2].y), f32x2_to_bf16x2(f.p[3].x, f.p[3].y));
        else
            q = make_uint4(__float_as_uint(f.p[(2 * v) % 4].x), __float_as_uint(f.p[(2 * v) % 4].y),
                           __float_as_uint(f.p[(2 * v + 1) % 4].x), __float_as_uint(f.p[(2 * v + 1) % 4].y));
        *reinterpret_cast<uint4 *>(static_cast<char *>(row) + l.at[v]) = q;
    }
}

/* Sum of the squares of the items that exist. */
template <int DT, bool VEC>
__device__ __forceinline__ float squares(const Items &f, const Lane<DT, VEC> &l)
{
    if (VEC && Lane<DT, VEC>::NV == 2) {
        const float2 a = __ffma2_rn(f.p[1], f.p[1], __fmul2_rn(f.p[0], f.p[0])), b = __ffma2_rn(f.p[3], f.p[3], __fmul2_rn(f.p[2], f.p[2]));
        return (l.in[0] ? a.x + a.y : 0.0f) + (l.in[Lane<DT, VEC>::NV - 1] ? b.x + b.y : 0.0f);
    }
    float2 q = __fmul2_rn(f.p[0], f.p[0]);
#pragma unroll
    for (int j = 1; j < kItems / 2; ++j) q = __ffma2_rn(f.p[j], f.p[j], q);
    return VEC && !l.in[0] ? 0.0f : q.x + q.y;
}

/* The same for binary32 arrays beside rows of either type (sums over rows). */
template <int DT, bool VEC>
__device__ __forceinline__ void store_f32(float *row, const Items &f, const Columns<DT, VEC> &c)
{
    const bool wide = VEC && ((uintptr_t)row & 15u) == 0;
#pragma unroll
    for (int j = 0; j < kItems; j += 4) {
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
 * would wait for the rows' stores as well.  CTAs of a cluster run at the same time, so the wait ends; its limit is
 * there for the case that it does not: the sum is NaN then.
 */
template <int N> struct RowSum {
    float4 warps[2][N][kMaxRowThreads / 32]; /* [turn][value][row of the CTA * vectors per row]: a word per warp, 0 behind the last */
    unsigned long long parts[2][N][kMaxNormCluster];
};
constexpr int kPartPolls = 1 << 22;
__host__ __device__ inline uint32_t sum_vectors(uint32_t tx) { return (tx / 32 + 3) / 4; }

/* Before the first row_sums; a barrier (of the cluster) must follow. */
template <int N> __device__ __forceinline__ void clear_row_sum(RowSum<N> &s)
{
    static_assert(sizeof(RowSum<N>) % 16 == 0, "cleared by vectors");
    for (uint32_t i = threadIdx.y * blockDim.x + threadIdx.x; i < sizeof s / 16; i += blockDim.x * blockDim.y)
        reinterpret_cast<float4 *>(&s)[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}

struct RowPlace {
    uint32_t tx, t, row, parts, part;        /* threads of a row, which of them, row of the CTA, CTAs of a row, which of them */
};

/* `call` counts the calls from 0. */
template <int N> __device__ __forceinline__ void row_sums(float (&v)[N], RowSum<N> &s, uint32_t call, const RowPlace &p)
{
    const uint32_t turn = call & 1u;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = warp_sum(v[k]);
    if (p.tx > 32) {
        const uint32_t n = sum_vectors(p.tx);
        if ((p.t & 31u) == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) reinterpret_cast<float *>(&s.warps[turn][k][p.row * n])[p.t / 32] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float4 *w = &s.warps[turn][k][p.row * n];
            float2 x = make_float2(0.0f, 0.0f);
#pragma unroll
            for (uint32_t i = 0; i < kMaxRowThreads / 128; ++i)
                if (i < n) { const float4 q = w[i]; x = __fadd2_rn(x, __fadd2_rn(make_float2(q.x, q.y), make_float2(q.z, q.w))); }
            v[k] = x.x + x.y;
        }
    }
    if (p.parts > 1) {
        if (p.t < p.parts) {
#pragma unroll
            for (int k = 0; k < N; ++k) store_cluster_tagged(&s.parts[turn][k][p.part], p.t, v[k], call + 1u);
        }
        int polls = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float x = 0.0f;
            for (uint32_t i = 0; i < p.parts; ++i) {
                unsigned long long w = load_tagged(&s.parts[turn][k][i]);
                while ((uint32_t)(w >> 32) != call + 1u && ++polls < kPartPolls) w = load_tagged(&s.parts[turn][k][i]);
                x += (uint32_t)(w >> 32) == call + 1u ? __uint_as_float((uint32_t)w) : NAN;
            }
            v[k] = x;
        }
    }
}

/* 1 / sqrt(mean + eps) */
__device__ __forceinline__ float rrms(float sum, uint32_t cols, float eps) { return rsqrtf(sum / (float)cols + eps); }

/*
 * Rows that are under way while others are worked on: a ring of shared memory that each thread fills with its own items
 * by asynchronous copies and reads itself, so that no barrier goes with it.  Place of (array k of a stage, word w of the
 * thread's Raw): words of the threads side by side, 16 bytes each (VEC) or 4.
 */
template <int DT, bool VEC> struct Ring {
    static constexpr bool possible = VEC || DT == SIFAR_F32;         /* a copy moves 4 bytes at least */
    static constexpr uint32_t bytes = sizeof(Raw<DT>);               /* per thread and array */
    static constexpr uint32_t unit = VEC ? 16 : 4;
    static constexpr int N = bytes / unit;
    uint32_t first, threads;                                         /* the thread's place in slot 0; of the CTA */
    uint32_t from[N], n[N];                                          /* of each copy: bytes into the row, bytes to move (the rest becomes 0) */
    __device__ __forceinline__ Ring(const void *smem, const Columns<DT, VEC> &c)
    {
        constexpr uint32_t es = sizeof(typename Elem<DT>::type);
        threads = blockDim.x * blockDim.y;
        first = (uint32_t)__cvta_generic_to_shared(smem) + (threadIdx.y * blockDim.x + threadIdx.x) * unit;
#pragma unroll
        for (int v = 0; v < N; ++v) {
            const uint32_t i = c.at(v * c.EPV);
            n[v] = i < c.cols ? min((uint32_t)c.EPV, c.cols - i) * es : 0u;
            from[v] = n[v] ? i * es : 0u;
        }
    }
    /* a row of an array to place `at` (bytes; a place takes `threads * bytes`) */
    __device__ __forceinline__ void fetch(uint32_t at, const void *row) const
    {
        const uint32_t to = first + at;
#pragma unroll
        for (int v = 0; v < N; ++v) {
            const char *p = static_cast<const char *>(row) + from[v];
            if (VEC)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to + v * threads * unit), "l"(p), "r"(n[v]) : "memory");
            else
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(to + v * threads * unit), "l"(p), "r"(n[v]) : "memory");
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
    __device__ __forceinline__ void read(Raw<DT> &x, uint32_t from) const
    {
        const uint32_t at = first + from;
#pragma unroll
        for (int v = 0; v < N; ++v) {
            if (VEC)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(x.w[4 * v % (bytes / 4)]), "=r"(x.w[(4 * v + 1) % (bytes / 4)]), "=r"(x.w[(4 * v + 2) % (bytes / 4)]),
                               "=r"(x.w[(4 * v + 3) % (bytes / 4)]) : "r"(at + v * threads * unit) : "memory");
            else
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x.w[v % (bytes / 4)]) : "r"(at + v * threads * unit) : "memory");
        }
    }
};
constexpr uint32_t kMaxStages = 4;
constexpr size_t kRingBytes = 220 * 1024;    /* of the 227 KB a CTA may have */

/* Rows of block b: [block_start(b), block_start(b + 1)). */
__host__ __device__ inline uint32_t block_start(uint32_t rows, uint32_t blocks, uint32_t b)
{
    return (uint32_t)((unsigned long long)rows * b / blocks);
}
__host__ __device__ inline uint32_t block_of(uint32_t rows, uint32_t blocks, uint32_t row)
{
    return (uint32_t)((((unsigned long long)row + 1ull) * blocks - 1ull) / rows);
}

/* How many CTAs hold a row and how many threads of each; into how many blocks of consecutive rows the rows are cut and
   how many of them a CTA walks side by side. */
constexpr unsigned kNormCtas = 148;          /* one per SM: rows under way and sums over rows fill its memory and registers */
struct RowShape {
    unsigned tx, parts, ry;
    uint32_t blocks;
};
inline RowShape row_shape(size_t rows, size_t cols)
{
    const size_t need = (cols + kItems - 1) / kItems;
    RowShape s;
    s.parts = 1;
    while ((need + s.parts - 1) / s.parts > (size_t)kMaxRowThreads) s.parts *= 2;
    s.tx = (unsigned)(((need + s.parts - 1) / s.parts + 31) / 32 * 32);
    s.ry = kMaxRowThreads / s.tx;
    while (s.ry > 1 && rows <= (size_t)(s.ry - 1) * kNormCtas) --s.ry;
    const size_t most = (size_t)(kNormCtas / s.parts) * s.ry;
    s.blocks = (uint32_t)(rows < most ? rows : most);
    return s;
}

/* Launches a kernel of blocks of rows with its ring; the attribute for that much shared memory is set once per kernel
   and device. */
template <int DT, bool VEC, typename Args>
cudaError_t launch_rows(void (*kernel)(Args), std::atomic<unsigned long long> &ready, const RowShape &sh, unsigned arrays,
                        cudaStream_t stream, Args &a)
{
    const size_t row = (size_t)sh.tx * sh.ry * arrays * Ring<DT, VEC>::bytes;
    const size_t turns = (a.rows + sh.blocks - 1) / sh.blocks;
    size_t stages = 1, smem = 0;
    if (Ring<DT, VEC>::possible) {
        stages = kRingBytes / row < kMaxStages ? kRingBytes / row : kMaxStages;
        if (stages > turns) stages = turns;
        smem = row * stages;
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev > 63 || !(ready.load(std::memory_order_acquire) >> dev & 1ull)) {
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes);
            if (e != cudaSuccess) return e;
            if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_release);
        }
    }
    a.stages = (uint32_t)stages;
    const dim3 grid((sh.blocks + sh.ry - 1) / sh.ry * sh.parts), block(sh.tx, sh.ry);
    return launch_op(kernel, grid, block, sh.parts, smem, stream, a);
}

}  /* namespace sifar */
#endif
