/*
 * sifar_norm_grad.cu - backward pass of sifar_block_norm (see sifar.h).
 *
 * Two kernels.  The first walks the rows: a block of consecutive rows per CTA (cluster, or part of a CTA), each row
 * read once and held in registers while its two sums are taken, the gradients that are summed over rows kept in
 * registers from row to row and stored once per block.  The second adds the blocks' sums in order, so that the
 * result does not depend on which CTA was first.
 *
 * 8192 x 4096 bf16, two norms and a gate: 85 to 91 us by run with two ranks' partials (5.5 to 5.2 TB/s,
 * 0.84 to 0.79 of the measured copy; 2.5 us of it the second kernel), 102 us with four (5.95 TB/s, 0.91).  What bounds it
 * below that is instructions, in 16 warps per SM, which is what the sums over rows leave registers for; each tenth of them
 * that went brought 5 to 6 % of the time.
 */
#include "sifar_norm.cuh"

namespace sifar {

constexpr unsigned kSumWarps = 16;

struct NormGradArgs {
    const void *dy[kMaxRanks];
    const void *dh, *h, *z;
    const float *stats;
    const void *post_weight, *gate, *pre_weight;
    void *dx, *dresidual;
    float *dgate;
    float *sum_post, *sum_pre, *sum_gate;    /* workspace: [block][pitch], [block][pitch], [block][2][pitch]; or NULL */
    uint32_t ld_dy, ld_dh, ld_h, ld_z, ld_gate, ld_dx, ld_dresidual;         /* bytes between two rows */
    float alpha, beta, offset;
    uint32_t rows, cols, pitch, blocks, rows_per_gate, parts, stages;
    int P, post, pre;
    int narrow, odd_start;                   /* rows so short that a vector may reach over the one beside it; an array that does
                                                not start on 16 bytes */
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

/* beta * gate of a row */
template <typename F>
__device__ __forceinline__ Items<F> gate_factor(const NormGradArgs &a, const Columns<F> &c, const Lane<F> &l, uint32_t row)
{
    if (!a.gate) return all_items<F>(a.beta);
    Items<F> g = load_factor(static_cast<const char *>(a.gate) + (unsigned long long)(row / a.rows_per_gate) * a.ld_gate, 0.0f, c, l);
#pragma unroll
    for (int j = 0; j < g.N; ++j) g.p[j] = __fmul2_rn(g.p[j], both(a.beta));
    return g;
}

/*
 * End of the rows [begin, end) of a block that share a gate row, with acc = their sum of D * n1: it gives the gate's
 * gradient, beta * (post_weight + offset) * acc, and adds beta * gate * acc to the post weight's.
 * The gate's is final where all rows of the gate row are here.  Otherwise it is a part: place 0 of the block's two
 * where it holds the block's first row, else place 1.  The post weight's sum is kept in the block's place of the
 * workspace, not in registers: gate rows end seldom.
 */
template <typename F>
__device__ __forceinline__ void end_of_gate(const NormGradArgs &a, const Columns<F> &c, const Lane<F> &l, Items<F> &acc,
                                            uint32_t b, uint32_t first, uint32_t begin, uint32_t end)
{
    if (a.sum_post) {
        float *const place = a.sum_post + (size_t)b * a.pitch;
        Items<F> post = gate_factor(a, c, l, begin);
#pragma unroll
        for (int j = 0; j < acc.N; ++j) post.p[j] = __fmul2_rn(post.p[j], acc.p[j]);
        if (begin != first) {
#pragma unroll
            for (int j = 0; j < F::items; ++j)
                if (c.has(j)) { if (j & 1) post.p[j / 2].y += place[c.at(j)]; else post.p[j / 2].x += place[c.at(j)]; }
        }
        store_f32(place, post, c);
    }
    if (a.dgate) {
        const Items<F> w = load_factor(a.post_weight, a.offset, c, l);
#pragma unroll
        for (int j = 0; j < acc.N; ++j) acc.p[j] = __fmul2_rn(__fmul2_rn(acc.p[j], both(a.beta)), w.p[j]);
        const uint32_t g = begin / a.rows_per_gate;
        const unsigned long long g0 = (unsigned long long)g * a.rows_per_gate, g1 = g0 + a.rows_per_gate;
        const bool whole = begin == g0 && (end == g1 || end == a.rows);
        if (whole) store_f32(a.dgate + (size_t)g * a.cols, acc, c);
        else store_f32(a.sum_gate + ((size_t)b * 2 + (begin == first ? 0 : 1)) * a.pitch, acc, c);
    }
    acc = all_items<F>(0.0f);
}

/* What a row leaves between the pass that takes its sums and the one that uses them. */
template <typename F, int N> struct Pending {
    Items<F> D;                              /* dh + r2 * a */
    Raw<F> h, z;
    float r1, r2, sum[N];
};

/*
 * Both sums of a row in one pass.  With t = dh + r2 * a and f = beta * gate * (post_weight + offset) the second,
 * sum(f * n1 * D) with D = t - r2 * m2 * n2, is sum(f * n1 * t) - r2 * m2 * sum(f * n1 * n2), so that neither has to
 * wait for the other.
 * AHEAD: the pass over a row that takes its sums runs before the one that uses those of the row before it: what the sums
 * need to meet, a barrier and in a cluster a word from every CTA, passes while there is other work.
 */
/* RANKS: that many partials, or 0: any number. */
template <typename F, bool POST, bool PRE, bool AHEAD, int RANKS>
__global__ void __launch_bounds__(kMaxRowThreads, 1) k_block_norm_grad(const __grid_constant__ NormGradArgs a)
{
    constexpr int kSums = POST && PRE ? 3 : 1;
    /* shifted rows: copied ahead in clusters (4096 x 4097, four ranks: 227 -> 185 us), read from memory, their lines asked
       for two rows before, where a CTA holds them (16384 x 515: 73 us against 86 with copies) */
    constexpr bool kRing = F::ACCESS != kShifted || AHEAD;
    extern __shared__ __align__(16) unsigned char ring_bytes[];
    __shared__ __align__(16) RowSum<kSums> s;
    grid_let_next_in();
    const RowPlace p{blockDim.x, threadIdx.x, threadIdx.y, a.parts, a.parts > 1 ? cluster_rank() : 0u};
    clear_row_sum(s);
    __syncthreads();
    if (a.parts > 1) { cluster_arrive(); cluster_wait(); }           /* all CTAs of the cluster have started */
    /* rows of more than a warp have their CTA to themselves: blocks never meet in a barrier */
    const uint32_t b = (blockIdx.x / a.parts) * blockDim.y + threadIdx.y;
    const bool live = b < a.blocks;
    const uint32_t first = live ? block_start(a.rows, a.blocks, b) : 0u, end = live ? block_start(a.rows, a.blocks, b + 1) : 0u;
    const Columns<F> c(p.part, p.tx, p.t, a.cols);
    const Lane<F> l(c);
    const Ring<F> ring(ring_bytes, c);
    const int partials = !PRE ? 0 : RANKS ? RANKS : a.P;
    const bool with_z = POST || a.z;
    const uint32_t pitch = ring.threads * ring.bytes;
    const uint32_t stage_bytes = pitch * ((uint32_t)partials + (PRE ? 1u : 0u) + (a.dh ? 1u : 0u) + (with_z ? 1u : 0u));
    grid_wait();

    /* rows that are read by elements when their turn comes: where a copy might reach over the array's start */
    const auto direct = [&](uint32_t row) {
        return Ring<F>::shifted && (a.narrow || (row == 0 && a.odd_start));
    };
    /* row `row` to place `to` of the ring: the partials, then h, dh, z */
    auto fetch = [&](uint32_t to, uint32_t row) {
        if (row < end && !direct(row)) {
            const unsigned long long at = row;
            if (PRE) {
                const unsigned long long o = at * a.ld_dy;
#pragma unroll (RANKS ? RANKS : 1)
                for (int r = 0; r < partials; ++r, to += pitch) ring.fetch(to, static_cast<const char *>(a.dy[r]) + o);
                ring.fetch(to, static_cast<const char *>(a.h) + at * a.ld_h);
                to += pitch;
            }
            if (a.dh) { ring.fetch(to, static_cast<const char *>(a.dh) + at * a.ld_dh); to += pitch; }
            if (with_z) ring.fetch(to, static_cast<const char *>(a.z) + at * a.ld_z);
        }
        ring.commit();
    };
    if (kRing)
        for (uint32_t i = 0; i < a.stages; ++i) fetch(i * stage_bytes, first + i);

    const Items<F> w2 = load_factor(a.pre_weight, a.offset, c, l);
    Items<F> f = load_factor(a.post_weight, a.offset, c, l);        /* of dx over D: post_weight + offset, beta, gate */
#pragma unroll
    for (int j = 0; j < f.N; ++j) f.p[j] = __fmul2_rn(f.p[j], both(a.beta));
    Items<F> pre = all_items<F>(0.0f), acc = pre;
    const float inv = 1.0f / (float)a.cols;
    uint32_t segment = first, gate_end = a.gate ? first : 0xFFFFFFFFu, place = 0;
    const uint32_t places = stage_bytes * a.stages;
    float next1 = POST && live ? a.stats[first] : 1.0f, next2 = PRE && live ? a.stats[a.rows + first] : 1.0f;

    auto take_sums = [&](Pending<F, kSums> &o, uint32_t row) {
        const unsigned long long at = row;
        o.r1 = next1;
        o.r2 = next2;
        if (row + 1 < end) {
            if (POST) next1 = a.stats[row + 1];
            if (PRE) next2 = a.stats[a.rows + row + 1];
        }
        if (kRing) ring.wait(a.stages - 1);
        float2 q2 = both(0.0f), qt = q2, qn = q2;         /* sums of a * n2, f * z * t, f * z * n2 */
        const auto pass = [&](bool each) {
#pragma unroll
            for (int v = 0; v < F::vectors; ++v) {            /* 16 bytes after 16 bytes: fewer registers */
                constexpr int N = F::vector_pairs;
                Raw<F> x, xd;
                float2 G[N];                                  /* the gradient of the normed h */
                const float2 before[3] = {q2, qt, qn};
                /* array k of the row in fetch's order */
                const auto get = [&](Raw<F> &y, int k, const void *base, uint32_t ld) {
                    const char *row_k = static_cast<const char *>(base) + at * ld;
                    if (kRing && !each) ring.read_vector(y, v, ring_bytes, place + (uint32_t)k * pitch, row_k);
                    else load_vector(y, v, row_k, c, l, each);
                };
                int k = partials;
                if (PRE) get(o.h, k++, a.h, a.ld_h);
                if (a.dh) get(xd, k++, a.dh, a.ld_dh);
                if (with_z) get(o.z, k, a.z, a.ld_z);
                if (PRE) {
                    get(x, 0, a.dy[0], a.ld_dy);
#pragma unroll
                    for (int j = 0; j < N; ++j) G[j] = pair<F>(x, v * N + j);
#pragma unroll (RANKS ? RANKS : 4)
                    for (int r = 1; r < partials; ++r) {
                        get(x, r, a.dy[r], a.ld_dy);
#pragma unroll
                        for (int j = 0; j < N; ++j) add_pair<F>(G[j], x, v * N + j);
                    }
                }
#pragma unroll
                for (int j = 0; j < N; ++j) o.D.p[v * N + j] = a.dh ? pair<F>(xd, v * N + j) : both(0.0f);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int i = v * N + j;
                    float2 n2;
                    if (PRE) {
                        n2 = __fmul2_rn(pair<F>(o.h, i), both(o.r2));
                        pre.p[i] = __ffma2_rn(G[j], n2, pre.p[i]);
                        G[j] = __fmul2_rn(G[j], w2.p[i]);
                        q2 = __ffma2_rn(G[j], n2, q2);
                        o.D.p[i] = __ffma2_rn(both(o.r2), G[j], o.D.p[i]);
                    }
                    if (POST) {
                        const float2 fz = __fmul2_rn(f.p[i], pair<F>(o.z, i));
                        qt = __ffma2_rn(fz, o.D.p[i], qt);
                        if (PRE) qn = __ffma2_rn(fz, n2, qn);
                    }
                }
                if (!kRing && F::VEC && !l.in[v]) { q2 = before[0]; qt = before[1]; qn = before[2]; }    /* nothing is 0 there */
            }
        };
        if (kRing ? direct(row) : by_element(l, row == 0 || row + 1 == a.rows || a.narrow)) pass(true);
        else pass(false);
        if (!kRing && row + 2 < end && (p.t & 7u) == 0) { /* a line of the row after next, into the L2 */
            const auto ahead = [&](const void *base, uint32_t ld) {
#pragma unroll
                for (int v = 0; v < F::vectors; ++v)
                    if (l.in[v]) asm volatile("prefetch.global.L2 [%0];" :: "l"(static_cast<const char *>(base) + (at + 2) * ld + l.at[v]));
            };
            if (PRE) {
                for (int r = 0; r < partials; ++r) ahead(a.dy[r], a.ld_dy);
                ahead(a.h, a.ld_h);
            }
            if (a.dh) ahead(a.dh, a.ld_dh);
            if (with_z) ahead(a.z, a.ld_z);
        }
        if (kRing) {
            fetch(place, row + a.stages);                 /* the thread has read its places */
            place = place + stage_bytes == places ? 0u : place + stage_bytes;
        }
        o.sum[0] = PRE ? q2.x + q2.y : qt.x + qt.y;
        if (kSums == 3) { o.sum[1 % kSums] = qt.x + qt.y; o.sum[2 % kSums] = qn.x + qn.y; }
        if (POST || PRE) publish_sums(o.sum, s, row - first, p);
    };

    auto use_sums = [&](Pending<F, kSums> &o, uint32_t row) {
        const unsigned long long at = row;
        Items<F> &D = o.D;                                /* from here on the gradient of h */
        if (POST || PRE) collect_sums(o.sum, s, row - first, p);
        const float m2 = PRE ? o.r2 * (o.sum[0] * inv) : 0.0f;
        const float m1 = !POST ? 0.0f : o.r1 * ((PRE ? o.sum[1 % kSums] - m2 * o.sum[2 % kSums] : o.sum[0]) * inv);
        if (PRE) {
#pragma unroll
            for (int j = 0; j < D.N; ++j) D.p[j] = __ffma2_rn(both(-m2 * o.r2), pair<F>(o.h, j), D.p[j]);
        }
        if (a.dresidual) {
            Items<F> r;
#pragma unroll
            for (int j = 0; j < D.N; ++j) r.p[j] = __fmul2_rn(both(a.alpha), D.p[j]);
            store_items(static_cast<char *>(a.dresidual) + at * a.ld_dresidual, r, c, l);
        }
        if (with_z) {
#pragma unroll
            for (int j = 0; j < D.N; ++j) {
                const float2 n1 = POST ? __fmul2_rn(pair<F>(o.z, j), both(o.r1)) : pair<F>(o.z, j);
                acc.p[j] = __ffma2_rn(D.p[j], n1, acc.p[j]);
                D.p[j] = __fmul2_rn(f.p[j], D.p[j]);
                if (POST) D.p[j] = __fmul2_rn(both(o.r1), __ffma2_rn(both(-m1), n1, D.p[j]));
            }
        } else {
#pragma unroll
            for (int j = 0; j < D.N; ++j) D.p[j] = __fmul2_rn(f.p[j], D.p[j]);
        }
        if (a.dx) store_items(static_cast<char *>(a.dx) + at * a.ld_dx, D, c, l);
    };

    auto gate_of = [&](uint32_t row) {                    /* the rows of another gate row begin */
        segment = row;
        gate_end = (row / a.rows_per_gate + 1) * a.rows_per_gate;
        f = load_factor(a.post_weight, a.offset, c, l);
        const Items<F> g = gate_factor(a, c, l, row);
#pragma unroll
        for (int j = 0; j < f.N; ++j) f.p[j] = __fmul2_rn(f.p[j], g.p[j]);
    };

    if (!AHEAD) {
        for (uint32_t row = first; row < end; ++row) {
            if (row >= gate_end) {
                if (row != first) end_of_gate(a, c, l, acc, b, first, segment, row);
                gate_of(row);
            }
            Pending<F, kSums> now;
            take_sums(now, row);
            if ((POST || PRE) && p.tx > 32) __syncthreads();
            if ((POST || PRE) && p.parts > 1) send_sums(s, row - first, p);
            use_sums(now, row);
        }
    } else {
        Pending<F, kSums> last;                           /* of row - 1, if `pending` */
        bool pending = false;
        for (uint32_t row = first; live; ++row) {
            if (pending && p.parts > 1 && (POST || PRE)) send_sums(s, row - 1 - first, p);
            if (row < end && row >= gate_end) {
                if (pending) {
                    use_sums(last, row - 1);
                    pending = false;
                    end_of_gate(a, c, l, acc, b, first, segment, row);
                }
                gate_of(row);
            }
            Pending<F, kSums> now;
            if (row < end) take_sums(now, row);
            if (pending) use_sums(last, row - 1);
            if (row >= end) break;
            last = now;
            pending = true;
            if (p.tx > 32) __syncthreads();
        }
    }
    if (kRing) ring.wait(0);
    if (!live) return;
    end_of_gate(a, c, l, acc, b, first, segment, end);
    if (a.sum_pre) store_f32(a.sum_pre + (size_t)b * a.pitch, pre, c);
}

struct NormSumArgs {
    const float *sum_post, *sum_pre, *sum_gate;
    float *dpost_weight, *dpre_weight, *dgate;
    uint32_t rows, cols, pitch, blocks, rows_per_gate, gates, gate_jobs, gate_warps, first_job, narrow;
};

/*
 * 32 columns per CTA, its warps over the blocks: part 0 is the post weight, 1 the pre weight, from 2 on the gate
 * rows that lie in more than one block, `gate_warps` warps each.  A gate row has a few blocks, a weight all of them:
 * with all warps on one gate row at a time 17 gate rows of 1003 x 4099 took 11 us.
 * Short rows have few columns and many blocks: a warp takes 8 columns of 4 blocks then (narrow).
 */
__global__ void __launch_bounds__(32 * kSumWarps) k_block_norm_sums(const __grid_constant__ NormSumArgs a)
{
    __shared__ float s[kSumWarps][32];
    grid_let_next_in();
    grid_wait();
    const uint32_t warp = threadIdx.y, lane = threadIdx.x, width = a.narrow ? 8u : 32u, subs = a.narrow ? 4u : 1u;
    const uint32_t col = blockIdx.x * width + (lane & (width - 1u)), sub = a.narrow ? lane >> 3 : 0u;
    const uint32_t part = blockIdx.y + a.first_job;
    const uint32_t warps = part < 2 ? kSumWarps : a.gate_warps, team = warps * subs, member = (warp % warps) * subs + sub;
    const float *p = nullptr;                             /* of the member's blocks; the first one may lie elsewhere */
    float *out = nullptr;
    size_t step = a.pitch;
    uint32_t n = 0;
    float v = 0.0f;
    if (part < 2) {
        p = part == 0 ? a.sum_post : a.sum_pre;
        out = part == 0 ? a.dpost_weight : a.dpre_weight;
        n = out ? a.blocks : 0u;
    } else {
        const uint32_t job = (part - 2) * (kSumWarps / warps) + warp / warps;
        /* more gate rows than blocks: one of them at most lies across the end of block `job` */
        const uint32_t g = a.gates < a.blocks || job + 1 >= a.blocks ? job : block_start(a.rows, a.blocks, job + 1) / a.rows_per_gate;
        if (job < a.gate_jobs && a.blocks == 0) {         /* no rows, one gate row for all of them: its gradient is 0 */
            out = a.dgate;
        } else if (job < a.gate_jobs) {
            const uint32_t r0 = g * a.rows_per_gate, r1 = a.rows - r0 > a.rows_per_gate ? r0 + a.rows_per_gate - 1 : a.rows - 1;
            const uint32_t b0 = block_of(a.rows, a.blocks, r0), b1 = block_of(a.rows, a.blocks, r1);
            /* within one block: already there; across several ends: the first end's */
            if (b0 != b1 && (a.gates < a.blocks || b0 == job)) {
                /* place 0 or 1 of the first block, place 0 of all others */
                n = b1 - b0 + 1;
                p = a.sum_gate + (size_t)b0 * 2 * a.pitch;
                step = 2 * (size_t)a.pitch;
                out = a.dgate + (size_t)g * a.cols;
                if (member == 0 && col < a.cols) {
                    const uint32_t place = block_start(a.rows, a.blocks, b0) == r0 ? 0u : 1u;
                    v = p[(size_t)place * a.pitch + col];
                }
            }
        }
    }
    if (out && col < a.cols) {
#pragma unroll 8
        for (uint32_t i = member + (part >= 2 && member == 0 ? team : 0u); i < n; i += team) v += p[i * step + col];
    }
    s[warp][lane] = v;
    __syncthreads();
    if (member == 0 && out && col < a.cols) {
        float x = 0.0f;
        for (uint32_t i = 0; i < warps; ++i)
            for (uint32_t k = 0; k < subs; ++k) x += s[warp + i][lane + k * width];
        out[col] = x;
    }
}

/* The attribute for the ring's shared memory is set once per kernel and device. */
template <typename F, bool POST, bool PRE, bool AHEAD, int RANKS>
static cudaError_t launch_grad_k(const GradShape &sh, unsigned arrays, cudaStream_t stream, NormGradArgs &a)
{
    static std::atomic<unsigned long long> ready{0};
    const auto kernel = k_block_norm_grad<F, POST, PRE, AHEAD, RANKS>;
    constexpr int kSums = POST && PRE ? 3 : 1;
    static_assert(sizeof(RowSum<kSums>) == row_sum_bytes(kSums), "what ring_room() leaves for the sums");
    size_t stages = 1, smem = 0;
    if (F::ACCESS != kShifted || AHEAD) {
        const size_t row = (size_t)sh.row.tx * sh.ry * arrays * Ring<F>::bytes;
        stages = grad_stages(sh, a.rows, row, kSums);
        smem = row * stages;
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev > 63 || !(ready.load(std::memory_order_acquire) >> dev & 1ull)) {
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ring_room(1, kSums));
            if (e != cudaSuccess) return e;
            if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_release);
        }
    }
    a.stages = (uint32_t)stages;
    const dim3 grid((sh.blocks + sh.ry - 1) / sh.ry * sh.row.parts), block(sh.row.tx, sh.ry);
    return launch_op(kernel, grid, block, sh.row.parts, smem, stream, a);
}

template <typename F, bool POST, bool PRE, int RANKS>
static cudaError_t launch_grad_r(bool ahead, const GradShape &sh, unsigned arrays, cudaStream_t stream, NormGradArgs &a)
{
    /* bf16 in clusters: a row ahead (2000 x 8200: 162 -> 124 us).  Without a cluster the barrier costs less than what the
       second row takes (8192 x 4096: 107 -> 115 us), fp32 has no registers for it (1003 x 4099: 50 -> 56 us). */
    if constexpr (F::DT == SIFAR_BF16)
        if (ahead) return launch_grad_k<F, POST, PRE, true, RANKS>(sh, arrays, stream, a);
    return launch_grad_k<F, POST, PRE, false, RANKS>(sh, arrays, stream, a);
}

template <int DT, Access A, bool POST, bool PRE>
static cudaError_t launch_grad_n(const GradShape &sh, unsigned arrays, cudaStream_t stream, NormGradArgs &a)
{
    using F = Form<DT, kGradWords<DT>, A>;
    const bool ahead = DT == SIFAR_BF16 && sh.row.parts > 1;
    /* loops over few partials cost as much as their work: one and two ranks have none (8192 x 4096 bf16, two: 98 -> 86 us),
       four in clusters (2000 x 8200: 140 -> 129; in CTAs 8192 x 4096 of four is at 102 us with the loop, at 106 without) */
    if constexpr (PRE && A == kWhole) {
        if (a.P == 1) return launch_grad_r<F, POST, PRE, 1>(ahead, sh, arrays, stream, a);
        if (a.P == 2) return launch_grad_r<F, POST, PRE, 2>(ahead, sh, arrays, stream, a);
        if constexpr (DT == SIFAR_BF16)
            if (a.P == 4 && ahead) return launch_grad_k<F, POST, PRE, true, 4>(sh, arrays, stream, a);
    }
    return launch_grad_r<F, POST, PRE, 0>(ahead, sh, arrays, stream, a);
}

template <int DT, Access A>
static cudaError_t launch_grad(const GradShape &sh, unsigned arrays, cudaStream_t stream, NormGradArgs &a)
{
    if (a.post) return a.pre ? launch_grad_n<DT, A, true, true>(sh, arrays, stream, a) : launch_grad_n<DT, A, true, false>(sh, arrays, stream, a);
    return a.pre ? launch_grad_n<DT, A, false, true>(sh, arrays, stream, a) : launch_grad_n<DT, A, false, false>(sh, arrays, stream, a);
}

/* Words between two blocks' sums. */
static size_t sum_pitch(size_t cols) { return (cols + 7) / 8 * 8; }

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
    const GradShape s = grad_shape(g->dtype, g->rows, g->cols);
    const size_t arrays = (g->dpost_weight ? 1 : 0) + (g->dpre_weight ? 1 : 0) + (g->dgate ? 2 : 0);
    return arrays * s.blocks * sum_pitch(g->cols) * sizeof(float);
}

extern "C" int sifar_block_norm_backward(const sifar_block_norm_grad_args *g, void *stream)
{
    static const char *fn = "sifar_block_norm_backward";
    if (int rc = check_grad_sizes(g, fn)) return rc;
    if (!std::isfinite(g->alpha) || !std::isfinite(g->beta) || !std::isfinite(g->weight_offset)) {
        set_error("%s: alpha, beta and weight_offset must be finite", fn);
        return SIFAR_ERR_INVALID;
    }
    /* without rows the arrays of rows have no element and may be NULL */
    if (g->rows && !g->dx && !g->dresidual && !g->dpost_weight && !g->dpre_weight && !g->dgate) {
        set_error("%s: no output is asked for", fn);
        return SIFAR_ERR_INVALID;
    }
    const bool post = g->post_norm != 0, pre = g->pre_norm != 0;
    if ((g->dpost_weight && !post) || (g->dpre_weight && !pre) || (g->dgate && !g->gate)) {
        set_error("%s: dpost_weight needs post_norm, dpre_weight pre_norm, dgate a gate", fn);
        return SIFAR_ERR_INVALID;
    }
    const bool need_z = post || g->dgate;
    if (g->rows && ((pre && !g->h) || (need_z && !g->z) || ((post || pre) && !g->stats) || (!pre && !g->dh))) {
        set_error("%s: h is needed with pre_norm, z with post_norm or dgate, stats with a norm, dh without pre_norm", fn);
        return SIFAR_ERR_INVALID;
    }
    const size_t rows = g->rows, cols = g->cols, es = elem_size(g->dtype);
    const size_t span = g->rows_per_gate && g->rows_per_gate < rows ? g->rows_per_gate : (rows ? rows : 1);
    /* one gate row for all rows is there without a row as well */
    const size_t gates = rows ? (rows + span - 1) / span : g->rows_per_gate ? 0 : 1;
    const size_t need = sifar_block_norm_backward_workspace(g);
    if (need && (!g->workspace || ((uintptr_t)g->workspace & 15u) || g->workspace_bytes < need)) {
        set_error("%s: need a 16-byte aligned workspace of %zu bytes", fn, need);
        return SIFAR_ERR_INVALID;
    }
    RowArray all[kMaxRanks + 16];
    int n = 0;
    for (int r = 0; pre && r < g->P; ++r) {
        if (rows && !g->dy[r]) { set_error("%s: dy[%d] is NULL", fn, r); return SIFAR_ERR_INVALID; }
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
    bool vec = rows_aligned16(dh), odd_start = false;
    for (int i = 0; i < n; ++i) {
        vec = vec && rows_aligned16(all[i]);
        odd_start = odd_start || ((uintptr_t)all[i].p & 15u) != 0;
    }
    odd_start = odd_start || ((uintptr_t)dh.p & 15u) != 0;
    if (post) all[n++] = RowArray{"post_weight", g->post_weight, 1, cols, cols, es, false};
    if (pre) all[n++] = RowArray{"pre_weight", g->pre_weight, 1, cols, cols, es, false};
    all[n++] = RowArray{"gate", g->gate, gates, cols, or_cols(g->ld_gate, cols), es, false};
    if (post || pre) all[n++] = RowArray{"stats", g->stats, 1, 2 * rows, 2 * rows, sizeof(float), false};
    all[n++] = RowArray{"dpost_weight", g->dpost_weight, 1, cols, cols, sizeof(float), true};
    all[n++] = RowArray{"dpre_weight", g->dpre_weight, 1, cols, cols, sizeof(float), true};
    all[n++] = RowArray{"dgate", g->dgate, gates, cols, cols, sizeof(float), true};
    if (need) all[n++] = RowArray{"workspace", g->workspace, 1, need / sizeof(float), need / sizeof(float), sizeof(float), true};
    if (int rc = check_arrays(fn, all, n)) return rc;

    const GradShape sh = grad_shape(g->dtype, rows, cols);
    float *ws = static_cast<float *>(g->workspace);
    const size_t plane = (size_t)sh.blocks * sum_pitch(cols);
    NormGradArgs a;
    for (int r = 0; r < kMaxRanks; ++r) a.dy[r] = pre && r < g->P ? g->dy[r] : nullptr;
    a.dh = g->dh; a.h = g->h; a.z = need_z ? g->z : nullptr; a.stats = g->stats;
    a.post_weight = post ? g->post_weight : nullptr; a.gate = g->gate; a.pre_weight = pre ? g->pre_weight : nullptr;
    a.dx = g->dx; a.dresidual = g->dresidual; a.dgate = g->dgate;
    a.sum_post = g->dpost_weight ? ws : nullptr; ws += g->dpost_weight ? plane : 0;
    a.sum_pre = g->dpre_weight ? ws : nullptr; ws += g->dpre_weight ? plane : 0;
    a.sum_gate = g->dgate ? ws : nullptr;
    const auto bytes = [&](size_t ld) { return (uint32_t)(or_cols(ld, cols) * es); };
    a.ld_dy = bytes(g->ld_dy); a.ld_dh = bytes(g->ld_dh); a.ld_h = bytes(g->ld_h); a.ld_z = bytes(g->ld_z);
    a.ld_gate = bytes(g->ld_gate); a.ld_dx = bytes(g->ld_dx); a.ld_dresidual = bytes(g->ld_dresidual);
    a.odd_start = odd_start;
    a.narrow = a.ld_dy < 32 || a.ld_dh < 32 || a.ld_h < 32 || a.ld_z < 32;
    a.alpha = g->alpha; a.beta = g->beta; a.offset = g->weight_offset;
    a.rows = (uint32_t)rows; a.cols = (uint32_t)cols; a.pitch = (uint32_t)sum_pitch(cols); a.blocks = sh.blocks;
    a.rows_per_gate = (uint32_t)span; a.parts = sh.row.parts;
    a.P = pre ? g->P : 1; a.post = post; a.pre = pre;
    if (rows) {
        const unsigned arrays = (pre ? (unsigned)g->P + 1u : 0u) + (g->dh ? 1u : 0u) + (need_z ? 1u : 0u);
        const cudaStream_t q = (cudaStream_t)stream;
        const cudaError_t err = g->dtype == SIFAR_BF16
            ? (vec ? launch_grad<SIFAR_BF16, kWhole>(sh, arrays, q, a) : launch_grad<SIFAR_BF16, kShifted>(sh, arrays, q, a))
            : (vec ? launch_grad<SIFAR_F32, kWhole>(sh, arrays, q, a) : launch_grad<SIFAR_F32, kElement>(sh, arrays, q, a));
        SIFAR_CUDA(err);
    }
    if (g->dpost_weight || g->dpre_weight || g->dgate) {
        NormSumArgs q;
        q.sum_post = a.sum_post; q.sum_pre = a.sum_pre; q.sum_gate = a.sum_gate;
        q.dpost_weight = g->dpost_weight; q.dpre_weight = g->dpre_weight; q.dgate = g->dgate;
        q.rows = a.rows; q.cols = a.cols; q.pitch = a.pitch; q.blocks = a.blocks; q.rows_per_gate = a.rows_per_gate;
        q.gates = g->dgate ? (uint32_t)gates : 0u;
        q.gate_warps = 1;
        while (q.gates && q.gate_warps < kSumWarps && q.blocks / q.gates >= 8 * q.gate_warps) q.gate_warps *= 2;
        const unsigned teams = kSumWarps / q.gate_warps;
        q.gate_jobs = q.gates < q.blocks || !q.blocks ? q.gates : q.blocks - 1;
        /* from the first part that is asked for to the last */
        q.first_job = q.dpost_weight ? 0u : q.dpre_weight ? 1u : 2u;
        const unsigned parts = q.gate_jobs ? 2 + (q.gate_jobs + teams - 1) / teams : q.dpre_weight ? 2u : 1u;
        q.narrow = cols <= 1024 && q.blocks >= 16 * kSumWarps;
        const unsigned width = q.narrow ? 8 : 32;
        const dim3 grid((unsigned)((cols + width - 1) / width), parts > q.first_job ? parts - q.first_job : 1u), block(32, kSumWarps);
        SIFAR_CUDA(launch_op(k_block_norm_sums, grid, block, 1, 0, (cudaStream_t)stream, q));
    }
    return SIFAR_OK;
}
