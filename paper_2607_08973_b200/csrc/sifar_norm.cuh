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
    float warps[2][kMaxRowThreads / 32];     /* [turn][row of the CTA * warps per row + warp] */
    float parts[2][kMaxNormCluster];
};

__device__ __forceinline__ float row_sum(float v, RowSum &s, int turn, uint32_t tx, uint32_t t, uint32_t row, uint32_t parts,
                                         uint32_t part)
{
    v = warp_sum(v);
    if (tx > 32) {
        const uint32_t n = tx / 32;
        float *w = &s.warps[turn][row * n];
        if ((t & 31u) == 0) w[t / 32] = v;
        __syncthreads();
        v = w[0];
        for (uint32_t i = 1; i < n; ++i) v += w[i];
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
