/*
 * How the norm kernels lay a row over threads, and the sum over a row.
 *
 * A thread holds kItems elements of a row in registers from its first load to its last store, so a row is read once
 * however many sums go over it.  A row takes `tx` threads of a CTA; where it is longer than kMaxRowThreads * kItems
 * elements, a cluster of up to eight CTAs holds it and its sums meet in their shared memory.
 */
#ifndef SIFAR_NORM_CUH
#define SIFAR_NORM_CUH

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

template <int DT> __device__ __forceinline__ float item(const Raw<DT> &x, int j)
{
    if (DT == SIFAR_BF16) return (j & 1) ? bf16hi_to_f32(x.w[j / 2]) : bf16lo_to_f32(x.w[j / 2]);
    return __uint_as_float(x.w[j % (sizeof x.w / 4)]);
}

/* acc[j] += item j, one binary32 add each */
template <int DT> __device__ __forceinline__ void add_items(float (&acc)[kItems], const Raw<DT> &x)
{
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        if (DT == SIFAR_BF16) acc[j] = (j & 1) ? add_bf16hi(acc[j], x.w[j / 2]) : add_bf16lo(acc[j], x.w[j / 2]);
        else acc[j] = __fadd_rn(acc[j], __uint_as_float(x.w[j % (sizeof x.w / 4)]));
    }
}

template <int DT, bool VEC>
__device__ __forceinline__ void store_row(void *row, const float (&f)[kItems], const Columns<DT, VEC> &c)
{
    using T = typename Elem<DT>::type;
    T *p = static_cast<T *>(row);
#pragma unroll
    for (int v = 0; v < Columns<DT, VEC>::NV; ++v) {
        const uint32_t i = c.at(v * c.EPV);
        if (VEC && i + c.EPV <= c.cols) {
            uint4 q;
            if (DT == SIFAR_BF16)
                q = make_uint4(f32x2_to_bf16x2(f[0], f[1]), f32x2_to_bf16x2(f[2], f[3]), f32x2_to_bf16x2(f[4], f[5]),
                               f32x2_to_bf16x2(f[6], f[7]));
            else
                q = make_uint4(__float_as_uint(f[(4 * v) % kItems]), __float_as_uint(f[(4 * v + 1) % kItems]),
                               __float_as_uint(f[(4 * v + 2) % kItems]), __float_as_uint(f[(4 * v + 3) % kItems]));
            *reinterpret_cast<uint4 *>(p + i) = q;
        } else {
#pragma unroll
            for (int k = 0; k < c.EPV; ++k)
                if (i + k < c.cols) p[i + k] = narrow<DT>(f[v * c.EPV + k]);
        }
    }
}

/* The same for binary32 arrays beside rows of either type (sums over rows). */
template <int DT, bool VEC>
__device__ __forceinline__ void store_f32(float *row, const float (&f)[kItems], const Columns<DT, VEC> &c)
{
    if (VEC && ((uintptr_t)row & 15u) == 0) {
#pragma unroll
        for (int j = 0; j < kItems; j += 4) {
            const uint32_t i = c.at(j);
            if (i + 4 <= c.cols) { *reinterpret_cast<float4 *>(row + i) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]); continue; }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < c.cols) row[i + k] = f[j + k];
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < kItems; ++j)
        if (c.has(j)) row[c.at(j)] = f[j];
}

/*
 * Sum of `v` over the threads of one row: warps by shuffles, a CTA's warps in order through shared memory, a
 * cluster's CTAs in rank order through its distributed shared memory.  All threads of the CTA (cluster) call it
 * together; `turn` alternates between calls, so that a fast warp does not overwrite what a slow one still reads.
 */
struct RowSum {
    float4 warps[2][kMaxRowThreads / 32];    /* [turn][row of the CTA * vectors per row]: a word per warp, 0 behind the last */
    float parts[2][kMaxNormCluster];
};
__host__ __device__ inline uint32_t sum_vectors(uint32_t tx) { return (tx / 32 + 3) / 4; }

/* Before the first row_sum; a barrier must follow. */
__device__ __forceinline__ void clear_row_sum(RowSum &s)
{
    const uint32_t i = threadIdx.y * blockDim.x + threadIdx.x;
    if (i < 2 * kMaxRowThreads / 32) (&s.warps[0][0])[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}

__device__ __forceinline__ float row_sum(float v, RowSum &s, int turn, uint32_t tx, uint32_t t, uint32_t row, uint32_t parts,
                                         uint32_t part)
{
    v = warp_sum(v);
    if (tx > 32) {
        const uint32_t n = sum_vectors(tx);
        float4 *w = &s.warps[turn][row * n];
        if ((t & 31u) == 0) reinterpret_cast<float *>(w)[t / 32] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < kMaxRowThreads / 128; ++i)
            if (i < n) { const float4 q = w[i]; v += (q.x + q.y) + (q.z + q.w); }
    }
    if (parts > 1) {
        if (t < parts) store_cluster_f32(&s.parts[turn][part], t, v);
        cluster_arrive();
        cluster_wait();
        v = s.parts[turn][0];
        for (uint32_t i = 1; i < parts; ++i) v += s.parts[turn][i];
    }
    return v;
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
    uint32_t base, threads, tid;
    __device__ __forceinline__ Ring(const void *smem)
        : base((uint32_t)__cvta_generic_to_shared(smem)), threads(blockDim.x * blockDim.y), tid(threadIdx.y * blockDim.x + threadIdx.x) {}
    __device__ __forceinline__ uint32_t place(uint32_t slot, int v) const
    {
        constexpr uint32_t unit = VEC ? 16 : 4;
        return base + ((slot * (bytes / unit) + (uint32_t)v) * threads + tid) * unit;
    }
    __device__ __forceinline__ void fetch(uint32_t slot, const void *row, const Columns<DT, VEC> &c) const
    {
        constexpr uint32_t es = sizeof(typename Elem<DT>::type);
        const char *p = static_cast<const char *>(row);
#pragma unroll
        for (int v = 0; v < Columns<DT, VEC>::NV; ++v) {
            const uint32_t i = c.at(v * c.EPV);
            const uint32_t n = i < c.cols ? min((uint32_t)c.EPV, c.cols - i) * es : 0u;      /* the rest becomes 0 */
            const char *from = n ? p + (size_t)i * es : p;
            if (VEC)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(place(slot, v)), "l"(from), "r"(n) : "memory");
            else
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(place(slot, v)), "l"(from), "r"(n) : "memory");
        }
    }
    __device__ __forceinline__ void commit() const { asm volatile("cp.async.commit_group;" ::: "memory"); }
    /* until all but the last n groups of this thread are there */
    __device__ __forceinline__ void wait(uint32_t n) const
    {
        if (n == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
        else if (n == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else if (n == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else asm volatile("cp.async.wait_group 3;" ::: "memory");
    }
    __device__ __forceinline__ void read(Raw<DT> &x, uint32_t slot) const
    {
#pragma unroll
        for (int v = 0; v < (int)(bytes / (VEC ? 16 : 4)); ++v) {
            if (VEC)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(x.w[4 * v % (bytes / 4)]), "=r"(x.w[(4 * v + 1) % (bytes / 4)]), "=r"(x.w[(4 * v + 2) % (bytes / 4)]),
                               "=r"(x.w[(4 * v + 3) % (bytes / 4)]) : "r"(place(slot, v)) : "memory");
            else
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x.w[v % (bytes / 4)]) : "r"(place(slot, v)) : "memory");
        }
    }
};
constexpr uint32_t kMaxStages = 4;
constexpr size_t kRingBytes = 220 * 1024;    /* of the 227 KB a CTA may have */

/* How many CTAs hold a row, and how many threads of each. */
struct RowShape {
    unsigned tx, parts;
};
inline RowShape row_shape(size_t cols)
{
    const size_t need = (cols + kItems - 1) / kItems;
    RowShape s;
    s.parts = 1;
    while ((need + s.parts - 1) / s.parts > (size_t)kMaxRowThreads) s.parts *= 2;
    s.tx = (unsigned)(((need + s.parts - 1) / s.parts + 31) / 32 * 32);
    return s;
}

}  /* namespace sifar */
#endif
