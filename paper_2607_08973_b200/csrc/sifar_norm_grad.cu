/*
 * sifar_norm_grad.cu - backward pass of sifar_block_norm (see sifar.h).
 *
 * Two kernels.  The first walks the rows: a block of consecutive rows per CTA (cluster, or part of a CTA), each row
 * read once and held in registers while its two sums are taken, the gradients that are summed over rows kept in
 * registers from row to row and stored once per block.  The second adds the blocks' sums in order, so that the
 * result does not depend on which CTA was first.
 */
#include <atomic>

#include "sifar_norm.cuh"

namespace sifar {

constexpr unsigned kGradCtas = 148;          /* one per SM: the row in flight and the sums over rows fill its registers */
constexpr unsigned kSumWarps = 16;

struct NormGradArgs {
    const void *dy[kMaxRanks];
    const void *dh, *h, *z;
    const float *stats;
    const void *post_weight, *gate, *pre_weight;
    void *dx, *dresidual;
    float *dgate;
    float *sum_post, *sum_pre, *sum_gate;    /* workspace: [block][pitch], [block][pitch], [block][2][pitch]; or NULL */
    unsigned long long ld_dy, ld_dh, ld_h, ld_z, ld_gate, ld_dx, ld_dresidual;    /* bytes between two rows */
    float alpha, beta, offset;
    uint32_t rows, cols, pitch, blocks, rows_per_gate, parts, stages;
    int P, post, pre;
};

/* Rows of block b: [block_start(b), block_start(b + 1)). */
__host__ __device__ inline uint32_t block_start(uint32_t rows, uint32_t blocks, uint32_t b)
{
    return (uint32_t)((unsigned long long)rows * b / blocks);
}
__host__ __device__ inline uint32_t block_of(uint32_t rows, uint32_t blocks, uint32_t row)
{
    return (uint32_t)((((unsigned long long)row + 1ull) * blocks - 1ull) / rows);
}

/*
 * The gate gradient of one gate row, as far as this block's rows [begin, end) go.  All rows of the gate row: the
 * final value.  Otherwise a part of it: place 0 of the block's two where it holds the block's first row, else place 1.
 */
template <int DT, bool VEC>
__device__ __forceinline__ void flush_gate(const NormGradArgs &a, const Columns<DT, VEC> &c, float (&acc)[kItems], uint32_t b,
                                           uint32_t first, uint32_t begin, uint32_t end)
{
    const uint32_t g = begin / a.rows_per_gate;
    const unsigned long long g0 = (unsigned long long)g * a.rows_per_gate, g1 = g0 + a.rows_per_gate;
    const bool whole = begin == g0 && (end == g1 || end == a.rows);
    if (whole) store_f32(a.dgate + (size_t)g * a.cols, acc, c);
    else store_f32(a.sum_gate + ((size_t)b * 2 + (begin == first ? 0 : 1)) * a.pitch, acc, c);
#pragma unroll
    for (int j = 0; j < kItems; ++j) acc[j] = 0.0f;
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(kMaxRowThreads, 1) k_block_norm_grad(const __grid_constant__ NormGradArgs a)
{
    extern __shared__ __align__(16) unsigned char ring_bytes[];
    __shared__ RowSum s;
    grid_let_next_in();
    const uint32_t tx = blockDim.x, t = threadIdx.x;
    const uint32_t part = a.parts > 1 ? cluster_rank() : 0u;
    clear_row_sum(s);
    __syncthreads();
    if (a.parts > 1) { cluster_arrive(); cluster_wait(); }
    const uint32_t b = (blockIdx.x / a.parts) * blockDim.y + threadIdx.y;
    const bool live = b < a.blocks;
    const uint32_t first = live ? block_start(a.rows, a.blocks, b) : 0u, end = live ? block_start(a.rows, a.blocks, b + 1) : 0u;
    const uint32_t turns = (a.rows + a.blocks - 1) / a.blocks;        /* the same for all threads: they meet in the sums */
    const Columns<DT, VEC> all(part, tx, t, a.cols);
    const Ring<DT, VEC> ring(ring_bytes);
    const uint32_t partials = a.pre ? (uint32_t)a.P : 0u, arrays = partials + (a.pre ? 1u : 0u) + (a.dh ? 1u : 0u) + (a.z ? 1u : 0u);
    grid_wait();

    /* row `row` into stage `stage`: the partials, then h, dh, z */
    auto fetch = [&](uint32_t stage, uint32_t row) {
        if (row < end) {
            uint32_t k = stage * arrays;
            for (uint32_t r = 0; r < partials; ++r) ring.fetch(k++, static_cast<const char *>(a.dy[r]) + row * a.ld_dy, all);
            if (a.pre) ring.fetch(k++, static_cast<const char *>(a.h) + row * a.ld_h, all);
            if (a.dh) ring.fetch(k++, static_cast<const char *>(a.dh) + row * a.ld_dh, all);
            if (a.z) ring.fetch(k++, static_cast<const char *>(a.z) + row * a.ld_z, all);
        }
        ring.commit();
    };
    if (Ring<DT, VEC>::possible)
        for (uint32_t i = 0; i < a.stages; ++i) fetch(i, first + i);

    Raw<DT> w1, w2;
    if (a.post_weight) load_any(w1, a.post_weight, all);
    if (a.pre_weight) load_any(w2, a.pre_weight, all);
    float acc1[kItems], acc2[kItems], accg[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) acc1[j] = acc2[j] = accg[j] = 0.0f;
    const float inv = 1.0f / (float)a.cols;
    uint32_t segment = first, stage = 0;
    int turn = 0;
    float next1 = a.post && live ? a.stats[first] : 1.0f, next2 = a.pre && live ? a.stats[a.rows + first] : 1.0f;

    for (uint32_t i = 0; i < turns; ++i) {
        const bool on = first + i < end;
        const uint32_t row = on ? first + i : 0u;
        const Columns<DT, VEC> c(part, tx, t, on ? a.cols : 0u);
        const float r1 = next1, r2 = next2;
        if (first + i + 1 < end) {
            if (a.post) next1 = a.stats[row + 1];
            if (a.pre) next2 = a.stats[a.rows + row + 1];
        }
        if (a.dgate && on && row != segment && row % a.rows_per_gate == 0) {
            flush_gate(a, all, accg, b, first, segment, row);
            segment = row;
        }
        Raw<DT> xg;
        if (a.gate) load_any(xg, static_cast<const char *>(a.gate) + (row / a.rows_per_gate) * a.ld_gate, c);

        float D[kItems], G[kItems];
        Raw<DT> xn, xz;
        if (Ring<DT, VEC>::possible) {
            ring.wait(a.stages - 1);
            uint32_t k = stage * arrays;
            if (a.pre) {
                Raw<DT> x;
                ring.read(x, k++);
#pragma unroll
                for (int j = 0; j < kItems; ++j) G[j] = item(x, j);
                for (uint32_t r = 1; r < partials; ++r) { ring.read(x, k++); add_items(G, x); }
                ring.read(xn, k++);
            }
            Raw<DT> x;
            if (a.dh) ring.read(x, k++);
#pragma unroll
            for (int j = 0; j < kItems; ++j) D[j] = a.dh ? item(x, j) : 0.0f;
            if (a.z) ring.read(xz, k);
            fetch(stage, first + i + a.stages);            /* the thread has read its places */
            stage = stage + 1 == a.stages ? 0u : stage + 1;
        } else {
            if (a.pre) {
                Raw<DT> x;
                load_row(x, static_cast<const char *>(a.dy[0]) + row * a.ld_dy, c);
#pragma unroll
                for (int j = 0; j < kItems; ++j) G[j] = item(x, j);
                for (uint32_t r = 1; r < partials; ++r) {
                    load_row(x, static_cast<const char *>(a.dy[r]) + row * a.ld_dy, c);
                    add_items(G, x);
                }
                load_row(xn, static_cast<const char *>(a.h) + row * a.ld_h, c);
            }
            Raw<DT> x;
            if (a.dh) load_row(x, static_cast<const char *>(a.dh) + row * a.ld_dh, c);
#pragma unroll
            for (int j = 0; j < kItems; ++j) D[j] = a.dh ? item(x, j) : 0.0f;
            if (a.z) load_row(xz, static_cast<const char *>(a.z) + row * a.ld_z, c);
        }
        if (!on) {                                         /* nothing was fetched for this thread */
#pragma unroll
            for (int j = 0; j < kItems; ++j) D[j] = G[j] = 0.0f;
            xn = xz = Raw<DT>{};
        }

        if (a.pre) {
            float q = 0.0f;
#pragma unroll
            for (int j = 0; j < kItems; ++j) {
                const float n2 = item(xn, j) * r2;
                acc2[j] = fmaf(G[j], n2, acc2[j]);
                if (a.pre_weight) G[j] *= item(w2, j) + a.offset;
                q = fmaf(G[j], n2, q);
            }
            const float m = row_sum(q, s, turn, tx, t, threadIdx.y, a.parts, part) * inv;
            turn ^= 1;
#pragma unroll
            for (int j = 0; j < kItems; ++j) D[j] = fmaf(r2, fmaf(-m, item(xn, j) * r2, G[j]), D[j]);
        }
        if (a.dresidual) {
            float o[kItems];
#pragma unroll
            for (int j = 0; j < kItems; ++j) o[j] = a.alpha * D[j];
            store_row(static_cast<char *>(a.dresidual) + row * a.ld_dresidual, o, c);
        }
        float q = 0.0f;
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            const float w = a.post && a.post_weight ? item(w1, j) + a.offset : 1.0f;
            const float n1 = a.z ? item(xz, j) * r1 : 0.0f;
            if (a.dgate) accg[j] = fmaf(a.beta * D[j], n1 * w, accg[j]);
            D[j] *= a.gate ? a.beta * item(xg, j) : a.beta;
            if (a.post) {
                acc1[j] = fmaf(D[j], n1, acc1[j]);
                D[j] *= w;
                q = fmaf(D[j], n1, q);
            }
        }
        if (a.post) {
            const float m = row_sum(q, s, turn, tx, t, threadIdx.y, a.parts, part) * inv;
            turn ^= 1;
#pragma unroll
            for (int j = 0; j < kItems; ++j) D[j] = r1 * fmaf(-m, item(xz, j) * r1, D[j]);
        }
        if (a.dx) store_row(static_cast<char *>(a.dx) + row * a.ld_dx, D, c);
    }
    if (Ring<DT, VEC>::possible) ring.wait(0);
    if (!live) return;
    if (a.sum_post) store_f32(a.sum_post + (size_t)b * a.pitch, acc1, all);
    if (a.sum_pre) store_f32(a.sum_pre + (size_t)b * a.pitch, acc2, all);
    if (a.dgate) flush_gate(a, all, accg, b, first, segment, end);
}

struct NormSumArgs {
    const float *sum_post, *sum_pre, *sum_gate;
    float *dpost_weight, *dpre_weight, *dgate;
    uint32_t rows, cols, pitch, blocks, rows_per_gate, gates;
};

/* 32 columns of a CTA: out[column] = the sum of `n` rows that are `step` floats apart. */
__device__ __forceinline__ void sum_blocks(const float *p, uint32_t n, size_t step, uint32_t col, uint32_t cols, float *out,
                                           float (*s)[32])
{
    float v = 0.0f;
    if (col < cols) {
#pragma unroll 4
        for (uint32_t i = threadIdx.y; i < n; i += kSumWarps) v += p[i * step + col];
    }
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y == 0 && col < cols) {
        for (uint32_t i = 1; i < kSumWarps; ++i) v += s[i][threadIdx.x];
        out[col] = v;
    }
    __syncthreads();
}

/* blockIdx.y = 0: post weight, 1: pre weight, from 2 on: the gate rows in turn. */
__global__ void __launch_bounds__(32 * kSumWarps) k_block_norm_sums(const NormSumArgs a)
{
    __shared__ float s[kSumWarps][32];
    grid_let_next_in();
    grid_wait();
    const uint32_t col = blockIdx.x * 32 + threadIdx.x;
    if (blockIdx.y == 0) {
        if (a.dpost_weight) sum_blocks(a.sum_post, a.blocks, a.pitch, col, a.cols, a.dpost_weight, s);
    } else if (blockIdx.y == 1) {
        if (a.dpre_weight) sum_blocks(a.sum_pre, a.blocks, a.pitch, col, a.cols, a.dpre_weight, s);
    } else {
        for (uint32_t g = blockIdx.y - 2; g < a.gates; g += gridDim.y - 2) {
            const unsigned long long last = min((unsigned long long)(g + 1ull) * a.rows_per_gate, (unsigned long long)a.rows) - 1;
            const uint32_t r0 = g * a.rows_per_gate;
            const uint32_t b0 = block_of(a.rows, a.blocks, r0), b1 = block_of(a.rows, a.blocks, (uint32_t)last);
            if (b0 == b1) continue;                       /* within one block: already there */
            /* place 0 or 1 of the first block, place 0 of all others */
            const uint32_t place = block_start(a.rows, a.blocks, b0) == r0 ? 0u : 1u;
            float v = 0.0f;
            if (col < a.cols)
                for (uint32_t i = threadIdx.y; i <= b1 - b0; i += kSumWarps)
                    v += a.sum_gate[((size_t)(b0 + i) * 2 + (i ? 0u : place)) * a.pitch + col];
            s[threadIdx.y][threadIdx.x] = v;
            __syncthreads();
            if (threadIdx.y == 0 && col < a.cols) {
                for (uint32_t i = 1; i < kSumWarps; ++i) v += s[i][threadIdx.x];
                a.dgate[(size_t)g * a.cols + col] = v;
            }
            __syncthreads();
        }
    }
}

/* Blocks of rows, and how many of them a CTA holds. */
struct GradShape {
    RowShape row;
    unsigned ry;
    uint32_t blocks;
    size_t pitch;
};
static GradShape grad_shape(size_t rows, size_t cols)
{
    GradShape s;
    s.row = row_shape(cols);
    s.ry = kMaxRowThreads / s.row.tx;
    while (s.ry > 1 && rows <= (size_t)(s.ry - 1) * kGradCtas) --s.ry;
    const size_t most = (size_t)(kGradCtas / s.row.parts) * s.ry;
    s.blocks = (uint32_t)(rows < most ? rows : most);
    s.pitch = (cols + kItems - 1) / kItems * kItems;
    return s;
}

/* The ring takes the shared memory that a CTA can have: the attribute is set once per kernel and device. */
template <int DT, bool VEC>
static cudaError_t launch_grad(dim3 grid, dim3 block, cudaStream_t stream, NormGradArgs &a, unsigned arrays)
{
    const size_t row = (size_t)block.x * block.y * arrays * Ring<DT, VEC>::bytes;
    size_t smem = 0;
    a.stages = 1;
    if (Ring<DT, VEC>::possible) {
        a.stages = (uint32_t)(kRingBytes / row < kMaxStages ? kRingBytes / row : kMaxStages);
        smem = row * a.stages;
    }
    static std::atomic<unsigned long long> ready{0};       /* a bit per device */
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (Ring<DT, VEC>::possible && (dev > 63 || !(ready.load(std::memory_order_acquire) >> dev & 1ull))) {
        e = cudaFuncSetAttribute(k_block_norm_grad<DT, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes);
        if (e != cudaSuccess) return e;
        if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_release);
    }
    return launch_op(k_block_norm_grad<DT, VEC>, grid, block, a.parts, smem, stream, a);
}

}  /* namespace sifar */

using namespace sifar;

static size_t or_cols(size_t ld, size_t cols) { return ld ? ld : cols; }

static int check_grad_sizes(const sifar_block_norm_grad_args *g, const char *fn)
{
    if (!g || (g->dtype != SIFAR_BF16 && g->dtype != SIFAR_F32) || (g->pre_norm && (g->P < 1 || g->P > kMaxRanks))) {
        set_error("%s: need an argument block with dtype in {0,1} and, with pre_norm, 1 <= P <= %d", fn, kMaxRanks);
        return SIFAR_ERR_INVALID;
    }
    if (g->cols < 1 || g->cols > SIFAR_NORM_MAX_COLS || g->rows >= kMaxRows) {
        set_error("%s: cols must be 1 .. %d and rows less than 2^31", fn, (int)SIFAR_NORM_MAX_COLS);
        return SIFAR_ERR_INVALID;
    }
    return SIFAR_OK;
}

extern "C" size_t sifar_block_norm_backward_workspace(const sifar_block_norm_grad_args *g)
{
    if (check_grad_sizes(g, "sifar_block_norm_backward_workspace")) return 0;
    const GradShape s = grad_shape(g->rows, g->cols);
    const size_t arrays = (g->dpost_weight ? 1 : 0) + (g->dpre_weight ? 1 : 0) + (g->dgate ? 2 : 0);
    return arrays * s.blocks * s.pitch * sizeof(float);
}

extern "C" int sifar_block_norm_backward(const sifar_block_norm_grad_args *g, void *stream)
{
    static const char *fn = "sifar_block_norm_backward";
    if (int rc = check_grad_sizes(g, fn)) return rc;
    if (!std::isfinite(g->alpha) || !std::isfinite(g->beta) || !std::isfinite(g->weight_offset)) {
        set_error("%s: alpha, beta and weight_offset must be finite", fn);
        return SIFAR_ERR_INVALID;
    }
    if (!g->dx && !g->dresidual && !g->dpost_weight && !g->dpre_weight && !g->dgate) {
        set_error("%s: no output is asked for", fn);
        return SIFAR_ERR_INVALID;
    }
    const bool post = g->post_norm != 0, pre = g->pre_norm != 0;
    if ((g->dpost_weight && !post) || (g->dpre_weight && !pre) || (g->dgate && !g->gate)) {
        set_error("%s: dpost_weight needs post_norm, dpre_weight pre_norm, dgate a gate", fn);
        return SIFAR_ERR_INVALID;
    }
    const bool need_z = post || g->dgate;
    if ((pre && !g->h) || (need_z && !g->z) || ((post || pre) && !g->stats) || (!pre && !g->dh)) {
        set_error("%s: h is needed with pre_norm, z with post_norm or dgate, stats with a norm, dh without pre_norm", fn);
        return SIFAR_ERR_INVALID;
    }
    const size_t rows = g->rows, cols = g->cols, es = elem_size(g->dtype);
    const size_t span = g->rows_per_gate && g->rows_per_gate < rows ? g->rows_per_gate : (rows ? rows : 1);
    const size_t gates = (rows + span - 1) / span, need = sifar_block_norm_backward_workspace(g);
    if (need && (!g->workspace || ((uintptr_t)g->workspace & 15u) || g->workspace_bytes < need)) {
        set_error("%s: need a 16-byte aligned workspace of %zu bytes", fn, need);
        return SIFAR_ERR_INVALID;
    }
    RowArray all[kMaxRanks + 16];
    int n = 0;
    for (int r = 0; pre && r < g->P; ++r) {
        if (!g->dy[r]) { set_error("%s: dy[%d] is NULL", fn, r); return SIFAR_ERR_INVALID; }
        all[n++] = RowArray{"dy", g->dy[r], rows, cols, or_cols(g->ld_dy, cols), es, false};
    }
    const RowArray dh{"dh", g->dh, rows, cols, or_cols(g->ld_dh, cols), es, false};
    const RowArray dres{"dresidual", g->dresidual, rows, cols, or_cols(g->ld_dresidual, cols), es, true};
    const bool in_place = g->dh && g->dh == g->dresidual && (dh.ld == dres.ld || rows <= 1);
    if (in_place) { if (int rc = check_array(fn, dh)) return rc; }
    else all[n++] = dh;
    all[n++] = dres;
    if (pre) all[n++] = RowArray{"h", g->h, rows, cols, or_cols(g->ld_h, cols), es, false};
    if (need_z) all[n++] = RowArray{"z", g->z, rows, cols, or_cols(g->ld_z, cols), es, false};
    all[n++] = RowArray{"dx", g->dx, rows, cols, or_cols(g->ld_dx, cols), es, true};
    bool vec = rows_aligned16(dh);
    for (int i = 0; i < n; ++i) vec = vec && rows_aligned16(all[i]);
    if (post) all[n++] = RowArray{"post_weight", g->post_weight, 1, cols, cols, es, false};
    if (pre) all[n++] = RowArray{"pre_weight", g->pre_weight, 1, cols, cols, es, false};
    all[n++] = RowArray{"gate", g->gate, gates, cols, or_cols(g->ld_gate, cols), es, false};
    if (post || pre) all[n++] = RowArray{"stats", g->stats, 1, 2 * rows, 2 * rows, sizeof(float), false};
    all[n++] = RowArray{"dpost_weight", g->dpost_weight, 1, cols, cols, sizeof(float), true};
    all[n++] = RowArray{"dpre_weight", g->dpre_weight, 1, cols, cols, sizeof(float), true};
    all[n++] = RowArray{"dgate", g->dgate, gates, cols, cols, sizeof(float), true};
    if (need) all[n++] = RowArray{"workspace", g->workspace, 1, need / sizeof(float), need / sizeof(float), sizeof(float), true};
    if (int rc = check_arrays(fn, all, n)) return rc;

    const GradShape sh = grad_shape(rows, cols);
    float *ws = static_cast<float *>(g->workspace);
    const size_t plane = (size_t)sh.blocks * sh.pitch;
    NormGradArgs a;
    for (int r = 0; r < kMaxRanks; ++r) a.dy[r] = pre && r < g->P ? g->dy[r] : nullptr;
    a.dh = g->dh; a.h = g->h; a.z = need_z ? g->z : nullptr; a.stats = g->stats;
    a.post_weight = post ? g->post_weight : nullptr; a.gate = g->gate; a.pre_weight = pre ? g->pre_weight : nullptr;
    a.dx = g->dx; a.dresidual = g->dresidual; a.dgate = g->dgate;
    a.sum_post = g->dpost_weight ? ws : nullptr; ws += g->dpost_weight ? plane : 0;
    a.sum_pre = g->dpre_weight ? ws : nullptr; ws += g->dpre_weight ? plane : 0;
    a.sum_gate = g->dgate ? ws : nullptr;
    a.ld_dy = or_cols(g->ld_dy, cols) * es; a.ld_dh = dh.ld * es; a.ld_h = or_cols(g->ld_h, cols) * es;
    a.ld_z = or_cols(g->ld_z, cols) * es; a.ld_gate = or_cols(g->ld_gate, cols) * es;
    a.ld_dx = or_cols(g->ld_dx, cols) * es; a.ld_dresidual = dres.ld * es;
    a.alpha = g->alpha; a.beta = g->beta; a.offset = g->weight_offset;
    a.rows = (uint32_t)rows; a.cols = (uint32_t)cols; a.pitch = (uint32_t)sh.pitch; a.blocks = sh.blocks;
    a.rows_per_gate = (uint32_t)span; a.parts = sh.row.parts;
    a.P = pre ? g->P : 1; a.post = post; a.pre = pre;
    if (rows) {
        const dim3 grid((sh.blocks + sh.ry - 1) / sh.ry * sh.row.parts), block(sh.row.tx, sh.ry);
        const unsigned arrays = (pre ? (unsigned)g->P + 1u : 0u) + (g->dh ? 1u : 0u) + (need_z ? 1u : 0u);
        const cudaStream_t q = (cudaStream_t)stream;
        const cudaError_t err = g->dtype == SIFAR_BF16 ? (vec ? launch_grad<SIFAR_BF16, true>(grid, block, q, a, arrays)
                                                              : launch_grad<SIFAR_BF16, false>(grid, block, q, a, arrays))
                                                       : (vec ? launch_grad<SIFAR_F32, true>(grid, block, q, a, arrays)
                                                              : launch_grad<SIFAR_F32, false>(grid, block, q, a, arrays));
        SIFAR_CUDA(err);
    }
    if (g->dpost_weight || g->dpre_weight || g->dgate) {
        NormSumArgs q;
        q.sum_post = a.sum_post; q.sum_pre = a.sum_pre; q.sum_gate = a.sum_gate;
        q.dpost_weight = g->dpost_weight; q.dpre_weight = g->dpre_weight; q.dgate = g->dgate;
        q.rows = a.rows; q.cols = a.cols; q.pitch = a.pitch; q.blocks = a.blocks; q.rows_per_gate = a.rows_per_gate;
        q.gates = g->dgate ? (uint32_t)gates : 0u;
        const unsigned gate_turns = q.gates < 64u ? q.gates : 64u;
        const dim3 grid((unsigned)((cols + 31) / 32), 2 + gate_turns), block(32, kSumWarps);
        SIFAR_CUDA(launch_op(k_block_norm_sums, grid, block, 1, 0, (cudaStream_t)stream, q));
    }
    return SIFAR_OK;
}
