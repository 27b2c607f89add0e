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
    uint32_t ld_x, ld_residual, ld_gate, ld_z, ld_h, ld_y;    /* bytes between two rows */
    float alpha, beta, eps, offset;
    uint32_t rows, cols, parts, rows_per_gate;
    int P, post, pre, narrow;                /* narrow: rows so short that a vector may reach over the one beside it */
};

/*
 * One row per threadIdx.y (and cluster).  All loads of a row go out before the first sum (where 64 bytes of an array lie
 * in a thread, as many partials as its registers take); z, h and y never leave the registers between.  PT is P or the
 * next power of two above it.
 *
 * Bound by memory where there are many rows: 8192 x 4096 bf16 of eight ranks, both norms and a gate, 118 to 127 us by
 * run = 6.2 to 5.8 TB/s, 0.95 to 0.89 of the measured copy; a row per CTA of 256 threads, two CTAs per SM (117
 * registers; four in the forms of 56 and 64), so that one's sums pass under the other's loads.  (One CTA per SM that walks its
 * rows with copies ahead: 124 to 130 us where this one took 118.)  Few ranks move less per row and thread: 8192 x 4096 bf16 of
 * one rank 47 us, 0.87.  Up to a row per SM the launch and one pass of latencies: 3.2 to 4.1 us.
 */
/*
 * Registers per thread: as many as keep several CTAs on an SM.  What spills (ptxas, bytes of stores a thread): nothing for
 * eight ranks but 308 for their shifted rows, up to 128 in the forms of one to four.  8192 x 4096 fp32 of one rank: 105 us
 * with 64 (two CTAs of 512 threads) against 166 with 72 (one); bf16 47 against 54.  Rows that are put together or read by
 * elements gain down to 56 (4000 x 3001 fp32: 36 against 42 us).  Eight ranks' rows want them all (8192 x 4096 bf16: 118 us
 * against 142 with 104), but for shifted ones, whose loads would take twice as many: four partials at a time and 72
 * (4096 x 4097 of eight: 155 us against 333 with 128).
 */
template <typename F, int PT> constexpr int kNormRegisters =
    F::W > 8 ? 112 : PT <= 2 ? (F::ACCESS == kWhole ? 64 : 56) : PT <= 4 ? (F::ACCESS == kWhole ? 64 : 72) : F::ACCESS == kWhole ? 128 : F::ACCESS == kElement ? 104 : 72;

/* Partials that are under way at once. */
template <typename F, int PT> constexpr int kNormBatch = F::W > 8 ? (F::DT == SIFAR_BF16 ? 2 : 4) : F::ACCESS == kShifted && PT > 4 ? 4 : PT;

template <typename F, int PT, int REGS>
__global__ void __launch_bounds__(kMaxRowThreads) __maxnreg__(REGS) k_block_norm(const __grid_constant__ NormArgs a)
{
    __shared__ __align__(16) RowSum<1> s;
    grid_let_next_in();
    const RowPlace p{blockDim.x, threadIdx.x, threadIdx.y, a.parts, a.parts > 1 ? cluster_rank() : 0u};
    clear_row_sum(s);
    __syncthreads();
    if (a.parts > 1) cluster_arrive();                   /* a CTA's shared memory may be written once it has started */
    const uint32_t row = (blockIdx.x / a.parts) * blockDim.y + threadIdx.y;
    const bool live = row < a.rows;
    const Columns<F> c(p.part, p.tx, p.t, live ? a.cols : 0u);
    const Lane<F> l(c);
    const unsigned long long at = live ? row : 0u;
    const bool edge = at == 0 || at + 1 >= a.rows || a.narrow;
    grid_wait();

    constexpr int B = kNormBatch<F, PT>;
    Raw<F> res, rg, rw1, rw2;
    Items<F> f;
    const char *gate = nullptr;
    if (a.gate) gate = static_cast<const char *>(a.gate) + (unsigned long long)((uint32_t)at / a.rows_per_gate) * a.ld_gate;
#pragma unroll
    for (int r0 = 0; r0 < PT; r0 += B) {
        if (r0 >= a.P) break;
        Raw<F> x[B];
        const auto load = [&](bool each) {
#pragma unroll
            for (int r = 0; r < B; ++r)
                if (r0 + r < a.P) load_row(x[r], static_cast<const char *>(a.x[r0 + r]) + at * a.ld_x, c, l, each);
            if (r0 == 0 && a.residual) load_row(res, static_cast<const char *>(a.residual) + at * a.ld_residual, c, l, each);
        };
        if (by_element(l, edge)) load(true);
        else load(false);
        if (r0 == 0) {
            if (F::W == 8) {
                if (a.gate) load_weight(rg, gate, c, l);
                if (a.post_weight) load_weight(rw1, a.post_weight, c, l);
                if (a.pre_weight) load_weight(rw2, a.pre_weight, c, l);
            }
            f = items<F>(x[0]);
        }
#pragma unroll
        for (int r = r0 == 0 ? 1 : 0; r < B; ++r)
            if (r0 + r < a.P) add_items(f, x[r]);
    }
    if (a.parts > 1) cluster_wait();
    if (a.z) store_items(static_cast<char *>(a.z) + at * a.ld_z, f, c, l);

    float r1 = 1.0f, r2 = 1.0f;
    uint32_t call = 0;
    if (a.post) {
        float sum[1] = {squares(f, l)};
        row_sums(sum, s, call++, p);
        r1 = rrms(sum[0], a.cols, a.eps);
#pragma unroll
        for (int j = 0; j < f.N; ++j) f.p[j] = __fmul2_rn(f.p[j], both(r1));
        if (a.post_weight) {
            if (F::W > 8) load_weight(rw1, a.post_weight, c, l);
#pragma unroll
            for (int j = 0; j < f.N; ++j) f.p[j] = __fmul2_rn(f.p[j], __fadd2_rn(pair<F>(rw1, j), both(a.offset)));
        }
    }
    if (a.gate) {
        if (F::W > 8) load_weight(rg, gate, c, l);
#pragma unroll
        for (int j = 0; j < f.N; ++j) f.p[j] = __fmul2_rn(f.p[j], pair<F>(rg, j));
    }
#pragma unroll
    for (int j = 0; j < f.N; ++j) f.p[j] = __fmul2_rn(f.p[j], both(a.beta));
    if (a.residual) {
#pragma unroll
        for (int j = 0; j < f.N; ++j) f.p[j] = __ffma2_rn(both(a.alpha), pair<F>(res, j), f.p[j]);
    }
    if (a.h) store_items(static_cast<char *>(a.h) + at * a.ld_h, f, c, l);
    if (a.pre) {
        float sum[1] = {squares(f, l)};
        row_sums(sum, s, call++, p);
        r2 = rrms(sum[0], a.cols, a.eps);
        if (a.y) {
#pragma unroll
            for (int j = 0; j < f.N; ++j) f.p[j] = __fmul2_rn(f.p[j], both(r2));
            if (a.pre_weight) {
                if (F::W > 8) load_weight(rw2, a.pre_weight, c, l);
#pragma unroll
                for (int j = 0; j < f.N; ++j) f.p[j] = __fmul2_rn(f.p[j], __fadd2_rn(pair<F>(rw2, j), both(a.offset)));
            }
            store_items(static_cast<char *>(a.y) + at * a.ld_y, f, c, l);
        }
    }
    if (a.stats && live && p.t == 0 && p.part == 0) {
        a.stats[row] = r1;
        a.stats[a.rows + row] = r2;
    }
}

template <int DT, int W, int PT>
static cudaError_t launch_norm_p(bool vec, dim3 grid, dim3 block, unsigned cluster, cudaStream_t stream, const NormArgs &a)
{
    using V = Form<DT, W, kWhole>;
    using E = Form<DT, W, DT == SIFAR_BF16 ? kShifted : kElement>;
    if (!vec) return launch_op(k_block_norm<E, PT, kNormRegisters<E, PT>>, grid, block, cluster, 0, stream, a);
    /* three and four ranks in fp32: 64 registers where two CTAs need it (4096 x 4096 of three: 80 us against 94 with 72), else
       72 (1003 x 4099, CTAs of 288 threads: 28 us against 33) */
    if constexpr (DT == SIFAR_F32 && W == 8 && PT == 4)
        if (block.x * block.y * 72 * 2 <= 65536) return launch_op(k_block_norm<V, PT, 72>, grid, block, cluster, 0, stream, a);
    return launch_op(k_block_norm<V, PT, kNormRegisters<V, PT>>, grid, block, cluster, 0, stream, a);
}

template <int DT>
static cudaError_t launch_norm(int words, bool vec, dim3 grid, dim3 block, unsigned cluster, cudaStream_t stream, const NormArgs &a)
{
    if (words == 16) return launch_norm_p<DT, 16, 8>(vec, grid, block, cluster, stream, a);
    if (a.P <= 1) return launch_norm_p<DT, 8, 1>(vec, grid, block, cluster, stream, a);
    if (a.P <= 2) return launch_norm_p<DT, 8, 2>(vec, grid, block, cluster, stream, a);
    if (a.P <= 4) return launch_norm_p<DT, 8, 4>(vec, grid, block, cluster, stream, a);
    return launch_norm_p<DT, 8, 8>(vec, grid, block, cluster, stream, a);
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
    if (g->y && !g->pre_norm) { set_error("%s: y needs pre_norm", fn); return SIFAR_ERR_INVALID; }
    if (g->rows == 0) return SIFAR_OK;                   /* arrays without an element may be NULL */
    if (!g->z && !g->h && !g->y) { set_error("%s: no output is asked for", fn); return SIFAR_ERR_INVALID; }

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
    a.residual = g->residual; a.gate = g->gate;
    a.post_weight = g->post_norm ? g->post_weight : nullptr; a.pre_weight = g->y ? g->pre_weight : nullptr;
    a.z = g->z; a.h = g->h; a.y = g->y; a.stats = g->stats;
    a.rows = (uint32_t)rows; a.cols = (uint32_t)cols;
    const auto bytes = [&](size_t ld) { return (uint32_t)(or_cols(ld, cols) * es); };
    a.ld_x = bytes(g->ld_x); a.ld_residual = bytes(g->ld_residual); a.ld_gate = bytes(g->ld_gate);
    a.ld_z = bytes(g->ld_z); a.ld_h = bytes(g->ld_h); a.ld_y = bytes(g->ld_y);
    a.rows_per_gate = (uint32_t)span;
    a.narrow = a.ld_x < 32 || a.ld_residual < 32;
    a.alpha = g->alpha; a.beta = g->beta; a.eps = g->eps; a.offset = g->weight_offset;
    a.P = g->P; a.post = g->post_norm != 0; a.pre = g->pre_norm != 0;
    /* 32 bytes of an array per thread; 64 where that keeps many rows out of clusters, whose sums cost more: 2000 x 8192
       fp32 104 -> 62 us, 4000 x 16384 bf16 220 -> 132 (four ranks: 245 -> 197).  Not where the row is just longer than a
       CTA (2000 x 4200 fp32: 39 against 47 us; from 9/8 on the 64 bytes win), not for more than four ranks (2000 x 8192
       fp32, eight: 131 against 147 us), not for few rows (one of 8192 fp32: 4.4 against 5.7 us). */
    const size_t cta = (size_t)kMaxRowThreads * 32 / es;
    const int words = rows > kSms && g->P <= 4 && cols > cta + cta / 8 && cols <= 2 * cta ? 16 : 8;
    const RowShape sh = row_shape(words * 4 / (int)es, cols);
    a.parts = sh.parts;
    /* short rows: several to a CTA once there is one for every SM */
    unsigned ry = 1;
    while (sh.parts == 1 && 2 * ry * sh.tx <= 256 && rows >= (size_t)2 * ry * 2 * kSms) ry *= 2;
    const unsigned long long grid = (rows + ry - 1) / ry * sh.parts;
    if (grid > 0x7FFFFFFFull) { set_error("%s: too many rows of this width", fn); return SIFAR_ERR_INVALID; }
    const dim3 gd((unsigned)grid), bd(sh.tx, ry);
    const cudaError_t err = g->dtype == SIFAR_BF16 ? launch_norm<SIFAR_BF16>(words, vec, gd, bd, sh.parts, (cudaStream_t)stream, a)
                                                   : launch_norm<SIFAR_F32>(words, vec, gd, bd, sh.parts, (cudaStream_t)stream, a);
    SIFAR_CUDA(err);
    return SIFAR_OK;
}
