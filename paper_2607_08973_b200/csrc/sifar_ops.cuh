/*
 * Shared by the operators behind an all-reduce (norms, routing): element access, sums over warps, CTAs and clusters
 * in a fixed order, launches, checks of arguments.
 */
#ifndef SIFAR_OPS_CUH
#define SIFAR_OPS_CUH

#include <cmath>

#include "sifar_internal.cuh"
#include "sifar_reduce.cuh"

namespace sifar {

/* ------------------------------------------------------------------------ */
/* device                                                                    */
/* ------------------------------------------------------------------------ */
template <int DT> struct Elem;
template <> struct Elem<SIFAR_BF16> { using type = uint16_t; static constexpr int per_vec = 8; };
template <> struct Elem<SIFAR_F32> { using type = uint32_t; static constexpr int per_vec = 4; };

template <int DT> __device__ __forceinline__ float widen(typename Elem<DT>::type v)
{
    return DT == SIFAR_BF16 ? __uint_as_float((uint32_t)v << 16) : __uint_as_float((uint32_t)v);
}
template <int DT> __device__ __forceinline__ typename Elem<DT>::type narrow(float f)
{
    if (DT == SIFAR_BF16) return (typename Elem<DT>::type)f32_to_bf16(f);
    return (typename Elem<DT>::type)__float_as_uint(f);
}

__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_let_next_in() { asm volatile("griddepcontrol.launch_dependents;"); }

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;                                          /* every lane adds the same pairs: the same bits in each */
}

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

/* A value and its tag in one 8-byte word: written into the same place of CTA `rank`'s shared memory, read from the own. */
__device__ __forceinline__ void store_cluster_tagged(unsigned long long *local, uint32_t rank, float v, uint32_t tag)
{
    const uint32_t a = (uint32_t)__cvta_generic_to_shared(local);
    const unsigned long long w = (unsigned long long)tag << 32 | __float_as_uint(v);
    asm volatile("{\n\t.reg .u32 q;\n\tmapa.shared::cluster.u32 q, %0, %1;\n\tst.relaxed.cluster.shared::cluster.b64 [q], %2;\n\t}"
                 :: "r"(a), "r"(rank), "l"(w) : "memory");
}
__device__ __forceinline__ unsigned long long load_tagged(const unsigned long long *local)
{
    unsigned long long w;
    asm volatile("ld.relaxed.cluster.shared::cta.b64 %0, [%1];" : "=l"(w) : "r"((uint32_t)__cvta_generic_to_shared(local)) : "memory");
    return w;
}

/* ------------------------------------------------------------------------ */
/* host                                                                      */
/* ------------------------------------------------------------------------ */
/* A kernel in clusters of `cluster` CTAs (1: none), its start overlapping the end of the kernel before it on the
   stream unless SIFAR_PDL=0 (it waits for that kernel before it reads anything). */
template <typename... Params, typename... Args>
cudaError_t launch_op(void (*kernel)(Params...), dim3 grid, dim3 block, unsigned cluster, size_t smem, cudaStream_t stream,
                      const Args &...args)
{
    cudaLaunchAttribute at[2];
    int n = 0;
    if (dependent_launches()) {
        at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        at[n].id = cudaLaunchAttributeClusterDimension;
        at[n].val.clusterDim.x = cluster;
        at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
        ++n;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.stream = stream; cfg.dynamicSmemBytes = smem;
    cfg.attrs = at; cfg.numAttrs = (unsigned)n;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

/* An array of `rows` rows of `cols` elements as an operator was given it. */
struct RowArray {
    const char *name;
    const void *p;
    size_t rows, cols, ld;            /* ld resolved: never 0 */
    size_t es;                        /* bytes per element */
    bool out;
};

constexpr size_t kMaxRows = (size_t)1 << 31;
constexpr size_t kMaxStride = ((size_t)1 << 30) - 1;      /* elements; in bytes it fits 32 bits */

/* Whether two arrays share an element.  Rows of one stride side by side in one buffer do not. */
inline bool share_elements(const RowArray &a, const RowArray &b)
{
    if (!a.p || !b.p || !a.rows || !b.rows || !a.cols || !b.cols) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    const size_t na = ((a.rows - 1) * a.ld + a.cols) * a.es, nb = ((b.rows - 1) * b.ld + b.cols) * b.es;
    if (!(x < y + nb && y < x + na)) return false;
    const size_t pitch = a.ld * a.es;
    if (pitch != b.ld * b.es) return true;
    const size_t wa = a.cols * a.es, wb = b.cols * b.es;
    const size_t shift = x <= y ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;     /* b's first column in a's row */
    return !(shift >= wa && shift + wb <= pitch);
}

/* Address, alignment and stride of one array; its text goes to sifar_last_error(). */
inline int check_array(const char *fn, const RowArray &a)
{
    if (!a.p) return SIFAR_OK;
    if ((uintptr_t)a.p % a.es) {
        set_error("%s: %s is not aligned to its %zu-byte elements", fn, a.name, a.es);
        return SIFAR_ERR_INVALID;
    }
    /* a list (ld = cols) is as long as it is: its kernels index it in 64 bits.  Rows have at most SIFAR_NORM_MAX_COLS columns */
    if (a.ld < a.cols || (a.ld > kMaxStride && a.ld != a.cols)) {
        set_error("%s: the row stride of %s (%zu) is less than its %zu columns, or too large", fn, a.name, a.ld, a.cols);
        return SIFAR_ERR_INVALID;
    }
    return SIFAR_OK;
}

/* Checks every array, and every output against all others; in-place pairs (the same address and stride) are the
   caller's to leave out. */
inline int check_arrays(const char *fn, const RowArray *a, int n)
{
    for (int i = 0; i < n; ++i)
        if (int rc = check_array(fn, a[i])) return rc;
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n; ++j)
            if ((a[i].out || a[j].out) && share_elements(a[i], a[j])) {
                set_error("%s: %s overlaps %s", fn, a[j].name, a[i].name);
                return SIFAR_ERR_INVALID;
            }
    return SIFAR_OK;
}

/* Whether all rows of an array start on a 16-byte boundary (one row: its stride does not matter). */
inline bool rows_aligned16(const RowArray &a)
{
    return !a.p || (((uintptr_t)a.p & 15u) == 0 && (a.rows <= 1 || (a.ld * a.es) % 16 == 0));
}

}  /* namespace sifar */
#endif
