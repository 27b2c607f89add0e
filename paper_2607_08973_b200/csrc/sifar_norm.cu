/*
 * sifar_norm.cu - the sum of P partials with the norms, gate and residual scale around a block (see sifar.h).
 */
#include "sifar_norm.cuh"

namespace sifar {

struct NormArgs {
    const void *x[kMaxRanks];
    const void *residual, *post_weight, *gate, *pre_weight;
    void *z, *h, *y;
    float *stats;
    unsigned long long rows;
    unsigned long long ld_x, ld_residual, ld_gate, ld_z, ld_h, ld_y;    /* bytes between two rows */
    float alpha, beta, eps, offset;
    uint32_t cols, parts, rows_per_gate;
    int P, post, pre;
};

/*
 * One row per threadIdx.y (and cluster).  All loads of a row go out before the first sum; z, h and y never leave the
 * registers between.  PT is P or the next power of two above it.
 */
template <int DT, int PT, bool VEC>
__global__ void __launch_bounds__(kMaxRowThreads) k_block_norm(const NormArgs a)
{
    __shared__ RowSum s;
    grid_let_next_in();
    const uint32_t tx = blockDim.x, t = threadIdx.x;
    const uint32_t part = a.parts > 1 ? cluster_rank() : 0u;
    if (a.parts > 1) cluster_arrive();                   /* a CTA's shared memory may be written once it has started */
    const unsigned long long row = (unsigned long long)(blockIdx.x / a.parts) * blockDim.y + threadIdx.y;
    const bool live = row < a.rows;
    const Columns<DT, VEC> c(part, tx, t, live ? a.cols : 0u);
    const unsigned long long at = live ? row : 0ull;
    clear_row_sum(s);
    __syncthreads();
    grid_wait();

    Raw<DT> x[PT], res, w1, w2, g;
#pragma unroll
    for (int r = 0; r < PT; ++r)
        if (r < a.P) load_row(x[r], static_cast<const char *>(a.x[r]) + at * a.ld_x, c);
    if (a.residual) load_row(res, static_cast<const char *>(a.residual) + at * a.ld_residual, c);
    if (a.post && a.post_weight) load_any(w1, a.post_weight, c);
    if (a.gate) load_any(g, static_cast<const char *>(a.gate) + (unsigned long long)((uint32_t)at / a.rows_per_gate) * a.ld_gate, c);
    if (a.pre && a.pre_weight) load_any(w2, a.pre_weight, c);
    if (a.parts > 1) cluster_wait();

    float f[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) f[j] = item(x[0], j);
#pragma unroll
    for (int r = 1; r < PT; ++r)
        if (r < a.P) add_items(f, x[r]);
    if (a.z) store_row(static_cast<char *>(a.z) + at * a.ld_z, f, c);

    float r1 = 1.0f, r2 = 1.0f;
    if (a.post) {
        float q = 0.0f;
#pragma unroll
        for (int j = 0; j < kItems; ++j) q = fmaf(f[j], f[j], q);
        r1 = rrms(row_sum(q, s, 0, tx, t, threadIdx.y, a.parts, part), a.cols, a.eps);
#pragma unroll
        for (int j = 0; j < kItems; ++j) f[j] *= a.post_weight ? r1 * (item(w1, j) + a.offset) : r1;
    }
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        f[j] *= a.gate ? a.beta * item(g, j) : a.beta;
        if (a.residual) f[j] = fmaf(a.alpha, item(res, j), f[j]);
        q = fmaf(f[j], f[j], q);
    }
    if (a.h) store_row(static_cast<char *>(a.h) + at * a.ld_h, f, c);
    if (a.pre) {
        r2 = rrms(row_sum(q, s, 1, tx, t, threadIdx.y, a.parts, part), a.cols, a.eps);
#pragma unroll
        for (int j = 0; j < kItems; ++j) f[j] *= a.pre_weight ? r2 * (item(w2, j) + a.offset) : r2;
        if (a.y) store_row(static_cast<char *>(a.y) + at * a.ld_y, f, c);
    }
    if (a.stats && live && t == 0 && part == 0) {
        a.stats[row] = r1;
        a.stats[a.rows + row] = r2;
    }
}

template <int DT, int PT>
static cudaError_t launch_norm_p(bool vec, dim3 grid, dim3 block, unsigned cluster, cudaStream_t stream, const NormArgs &a)
{
    return vec ? launch_op(k_block_norm<DT, PT, true>, grid, block, cluster, 0, stream, a)
               : launch_op(k_block_norm<DT, PT, false>, grid, block, cluster, 0, stream, a);
}

template <int DT>
static cudaError_t launch_norm(bool vec, dim3 grid, dim3 block, unsigned cluster, cudaStream_t stream, const NormArgs &a)
{
    if (a.P <= 1) return launch_norm_p<DT, 1>(vec, grid, block, cluster, stream, a);
    if (a.P <= 2) return launch_norm_p<DT, 2>(vec, grid, block, cluster, stream, a);
    if (a.P <= 4) return launch_norm_p<DT, 4>(vec, grid, block, cluster, stream, a);
    return launch_norm_p<DT, 8>(vec, grid, block, cluster, stream, a);
}

}  /* namespace sifar */

using namespace sifar;

static size_t or_cols(size_t ld, size_t cols) { return ld ? ld : cols; }

extern "C" int sifar_block_norm(const sifar_block_norm_args *g, void *stream)
{
    static const char *fn = "sifar_block_norm";
    if (!g || g->P < 1 || g->P > kMaxRanks || (g->dtype != SIFAR_BF16 && g->dtype != SIFAR_F32)) {
        set_error("%s: need an argument block with 1 <= P <= %d and dtype in {0,1}", fn, kMaxRanks);
        return SIFAR_ERR_INVALID;
    }
    if (g->cols < 1 || g->cols > SIFAR_NORM_MAX_COLS || g->rows >= kMaxRows) {
        set_error("%s: cols must be 1 .. %d and rows less than 2^31", fn, (int)SIFAR_NORM_MAX_COLS);
        return SIFAR_ERR_INVALID;
    }
    if (!std::isfinite(g->alpha) || !std::isfinite(g->beta) || !std::isfinite(g->weight_offset) || !std::isfinite(g->eps) ||
        g->eps < 0.0f) {
        set_error("%s: alpha, beta, weight_offset and eps must be finite, eps not negative", fn);
        return SIFAR_ERR_INVALID;
    }
    if (!g->z && !g->h && !g->y) { set_error("%s: no output is asked for", fn); return SIFAR_ERR_INVALID; }
    if (g->y && !g->pre_norm) { set_error("%s: y needs pre_norm", fn); return SIFAR_ERR_INVALID; }
    if (g->rows == 0) return SIFAR_OK;

    const size_t rows = g->rows, cols = g->cols, es = elem_size(g->dtype);
    const size_t span = g->rows_per_gate && g->rows_per_gate < rows ? g->rows_per_gate : rows, gates = (rows + span - 1) / span;
    RowArray all[kMaxRanks + 8];
    int n = 0;
    for (int r = 0; r < g->P; ++r) {
        if (!g->x[r]) { set_error("%s: x[%d] is NULL", fn, r); return SIFAR_ERR_INVALID; }
        all[n++] = RowArray{"x", g->x[r], rows, cols, or_cols(g->ld_x, cols), es, false};
    }
    const RowArray residual{"residual", g->residual, rows, cols, or_cols(g->ld_residual, cols), es, false};
    const RowArray h{"h", g->h, rows, cols, or_cols(g->ld_h, cols), es, true};
    const bool in_place = g->h && g->h == g->residual && (h.ld == residual.ld || rows == 1);
    if (in_place) { if (int rc = check_array(fn, residual)) return rc; }
    else all[n++] = residual;
    all[n++] = RowArray{"z", g->z, rows, cols, or_cols(g->ld_z, cols), es, true};
    all[n++] = h;
    all[n++] = RowArray{"y", g->y, rows, cols, or_cols(g->ld_y, cols), es, true};
    bool vec = rows_aligned16(residual);
    for (int i = 0; i < n; ++i) vec = vec && rows_aligned16(all[i]);
    all[n++] = RowArray{"post_weight", g->post_weight, 1, cols, cols, es, false};
    all[n++] = RowArray{"gate", g->gate, gates, cols, or_cols(g->ld_gate, cols), es, false};
    all[n++] = RowArray{"pre_weight", g->pre_weight, 1, cols, cols, es, false};
    all[n++] = RowArray{"stats", g->stats, 1, 2 * rows, 2 * rows, sizeof(float), true};
    if (int rc = check_arrays(fn, all, n)) return rc;

    NormArgs a;
    for (int r = 0; r < kMaxRanks; ++r) a.x[r] = r < g->P ? g->x[r] : nullptr;
    a.residual = g->residual; a.post_weight = g->post_weight; a.gate = g->gate; a.pre_weight = g->pre_weight;
    a.z = g->z; a.h = g->h; a.y = g->y; a.stats = g->stats;
    a.rows = rows; a.cols = (uint32_t)cols;
    a.ld_x = or_cols(g->ld_x, cols) * es; a.ld_residual = residual.ld * es; a.ld_gate = or_cols(g->ld_gate, cols) * es;
    a.ld_z = or_cols(g->ld_z, cols) * es; a.ld_h = h.ld * es; a.ld_y = or_cols(g->ld_y, cols) * es;
    a.rows_per_gate = (uint32_t)span;
    a.alpha = g->alpha; a.beta = g->beta; a.eps = g->eps; a.offset = g->weight_offset;
    a.P = g->P; a.post = g->post_norm != 0; a.pre = g->pre_norm != 0;
    const RowShape sh = row_shape(cols);
    a.parts = sh.parts;
    unsigned ry = 1;
    while (sh.parts == 1 && 2 * ry * sh.tx <= 256 && rows >= (size_t)2 * ry * 296) ry *= 2;
    const unsigned long long grid = (rows + ry - 1) / ry * sh.parts;
    if (grid > 0x7FFFFFFFull) { set_error("%s: too many rows of this width", fn); return SIFAR_ERR_INVALID; }
    const dim3 gd((unsigned)grid), bd(sh.tx, ry);
    const cudaError_t err = g->dtype == SIFAR_BF16 ? launch_norm<SIFAR_BF16>(vec, gd, bd, sh.parts, (cudaStream_t)stream, a)
                                                   : launch_norm<SIFAR_F32>(vec, gd, bd, sh.parts, (cudaStream_t)stream, a);
    SIFAR_CUDA(err);
    return SIFAR_OK;
}
