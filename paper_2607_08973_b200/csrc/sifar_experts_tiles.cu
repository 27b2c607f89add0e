/*
 * sifar_experts_tiles.cu - the chosen experts' products for more than a few tokens, bf16: tcgen05 matrix instructions on
 * tiles of up to 128 weight rows.
 *
 * The weights are the instruction's rows (M = 128) and an expert's tokens its columns (N = 16 .. 64), so that every weight is
 * read once whatever the number of tokens.  A stage of the ring in shared memory is 64 elements (128 bytes, a swizzle atom)
 * of the tile's rows and of the tokens' rows.  The warps of a CTA have parts of their own and meet only through the stages'
 * barriers:
 *   warp 0      fetches the weights (TMA, 128, 64, 32 and 16 rows at a time: no more than the share has)
 *   warp 1      issues the products
 *   warps 2, 3  gather the tokens' rows (asynchronous 16-byte copies)
 *   warps 4 - 11  take a tile's sums out of tensor memory while the next tile's go into its other half, each half of the columns
 * What bounds it is the memory (64 tokens that chose 70 experts of 768 x 4096: 236 us, 5.6 TB/s), and with many tokens per expert the
 * steps themselves (256 tokens on 24 experts: 128 us, 3.6 TB/s); the ring keeps up to 160 KB of weights per SM on the way, across tiles.  Warps 0 and 1 go through
 * their loops as whole warps and one lane issues: what an instruction of these needs is in uniform registers then (as one thread's
 * loop, a product took 150 cycles to issue and a fetch 90).
 *
 * First product: a tile is 128 gate rows and the 128 up rows that go with them, two accumulators; a thread then has both values of
 * its row.  Second product: the values come as two bf16 parts, and both go into one accumulator.
 */
#include <cstdlib>

#include <cuda.h>

#include "sifar_experts.cuh"

namespace sifar {

constexpr int kRows = 128;                   /* of an instruction */
constexpr int kSpan = 128;                   /* bytes of a row in a stage */
constexpr int kGroup = 16;                   /* rows that tiles are counted in, and that the smallest fetch of weights has */
constexpr int kGroups = kRows / kGroup;
constexpr int kRing = 204 * 1024;            /* bytes of all stages: what the lists leave of an SM's 227 KB */
constexpr int kMaxRing = 8;
constexpr int kTileWarps = 12, kTileThreads = 32 * kTileWarps, kDrainers = 8;
constexpr int kGatherers = 64;               /* threads that gather the tokens' rows */
constexpr int kLag = 3;                      /* stages that they have under way while they fill another: less than a ring has */
constexpr uint32_t kPolls = 1u << 22;        /* a wait's limit unless the environment has another: about 0.1 s, where the products take less than a microsecond */

template <bool DOWN> struct Tile {
    static constexpr int halves = DOWN ? 1 : 2;                  /* blocks of kRows weight rows */
    static constexpr int parts = DOWN ? 2 : 1;                   /* of the tokens' values */
};

struct TilesArgs {
    ExpertsArgs e;
    uint32_t columns;                        /* of a pass over an expert's rows */
    uint32_t polls;                          /* limit of a wait */
};

__device__ __forceinline__ uint32_t shared_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

/* Operand in shared memory: rows of 128 bytes in 128-byte swizzle, eight rows every 1024 bytes. */
__device__ __forceinline__ unsigned long long operand(uint32_t at)
{
    return (unsigned long long)((at & 0x3FFFFu) >> 4) | 1ull << 16 | (unsigned long long)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
/* These are gone through by a whole warp and issued by the lane whose `leader` is not 0. */
__device__ __forceinline__ uint32_t elect_leader()
{
    uint32_t leader;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(leader));
    return leader;
}
__device__ __forceinline__ void product(uint32_t leader, uint32_t to, unsigned long long rows, unsigned long long cols, uint32_t kind, bool add)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(to), "l"(rows), "l"(cols), "r"(kind), "r"((uint32_t)add), "r"(leader) : "memory");
}
/* The barrier is told when all products issued so far are done. */
__device__ __forceinline__ void tell_when_done(uint32_t leader, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                 :: "r"(bar), "r"(leader) : "memory");
}
__device__ __forceinline__ void sums_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void sums_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void read_sums(uint32_t (&v)[8], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(at));
}

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ void bar_arrive_and_expect(uint32_t leader, uint32_t bar, uint32_t bytes)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" :: "r"(bar), "r"(bytes), "r"(leader) : "memory");
}
/*
 * Whether the barrier's phase `parity` is over, the same for the whole warp; false where that takes too long.  A warp whose wait has
 * run out neither fills stages nor tells a barrier of anything any more, so the waits of those that depend on it run out too, and
 * what a barrier has told of is right.  The warps that take sums out leave NaN from then on.
 * UNIFORM: the answer comes by a shuffle from one lane, so that the compiler sees that it is the same for all and keeps what the
 * instructions behind it need in uniform registers (where it does not: 64 tokens 265 us, quarter 169).
 */
template <bool UNIFORM = false>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t polls)
{
    uint32_t i = 0;
    int all;
    do {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        all = __all_sync(0xFFFFFFFFu, done);
    } while (!all && i++ < polls);
    return UNIFORM ? __shfl_sync(0xFFFFFFFFu, all, 0) : all;
}

/* The map's number of rows x 64 elements from (column, row) on. */
__device__ __forceinline__ void fetch_rows(uint32_t leader, uint32_t to, const CUtensorMap *map, uint32_t column, uint32_t row, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %5, 0;\n\t"
                 "@q cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
                 :: "r"(to), "l"(map), "r"(column), "r"(row), "r"(bar), "r"(leader) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const char *from, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(bytes) : "memory");
}

/* With the short exponential and quotient: a few steps of binary32 off (e: 2, its argument: |x|, the quotient: 2), where 16 bits
   are kept.  A quotient by more than 2^126 is 0. */
__device__ __forceinline__ float activate_fast(float g, int kind)
{
    if (kind == SIFAR_ACT_SILU) return __fdividef(g, 1.0f + __expf(-g));
    return activate(g, kind);
}

/* A tile: rows row .. row + count - 1 of a pass over an expert with the tokens first .. first + n - 1 of the list. */
struct TileAt { uint32_t expert, row, count, first, n; };

/* The same rows, 128 >> i at a time. */
struct RowMaps { CUtensorMap of[4]; };

template <bool DOWN>
__global__ void __launch_bounds__(kTileThreads, 1) k_expert_tiles(const __grid_constant__ RowMaps maps, const __grid_constant__ TilesArgs ta)
{
    using S = Tile<DOWN>;
    const ExpertsArgs &a = ta.e;
    extern __shared__ __align__(1024) char smem[];                  /* the ring; at first each expert's tokens as bits */
    __shared__ uint16_t s_place[SIFAR_ROUTE_MAX_EXPERTS];           /* of an expert's first token in the list */
    __shared__ uint16_t s_list[SIFAR_ROUTE_MAX_EXPERTS];            /* experts that have tokens */
    __shared__ uint16_t s_first[SIFAR_ROUTE_MAX_EXPERTS + 1], s_passes[SIFAR_ROUTE_MAX_EXPERTS + 1];   /* tokens of the list, passes before each */
    __shared__ uint8_t s_token[SIFAR_EXPERTS_MAX_TOKENS * SIFAR_ROUTE_MAX_TOP_K];      /* the tokens by expert, in their order */
    __shared__ unsigned long long s_sum[kTileWarps];
    __shared__ __align__(8) unsigned long long s_full[kMaxRing], s_empty[kMaxRing], s_sums[2], s_free[2], s_done;
    __shared__ uint32_t s_tmem, s_told[kGatherers / 32];
    __shared__ __align__(16) float s_weight[kDrainers][32];         /* of a tile's tokens, each warp's half */
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    uint32_t *const s_bits = reinterpret_cast<uint32_t *>(smem);
    if (warp == 0 && lane < 4) asm volatile("prefetch.tensormap [%0];" :: "l"(&maps.of[lane]) : "memory");
    if (!DOWN) grid_wait();
    grid_let_next_in();                                             /* the choices are complete: the next kernel may read them too */

    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(shared_at(&s_tmem)), "r"(256u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        sums_before();
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxRing; ++i) {
            bar_init(shared_at(&s_full[i]), 1 + kGatherers / 32);
            bar_init(shared_at(&s_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(shared_at(&s_sums[i]), 1);
            bar_init(shared_at(&s_free[i]), kDrainers);
        }
        bar_init(shared_at(&s_done), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const ExpertPlan plan = plan_experts<kTileThreads>(a, [&](const auto &) { return ta.columns; }, s_bits, s_sum, s_place, s_list, s_first, s_passes, s_token, !DOWN && blockIdx.x == 0);
    sums_after();                                                   /* the address of tensor memory */
    const int active = plan.active;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    /* what was read and written where the ring is now */
    __syncthreads();
    const uint32_t tmem = s_tmem;

    /* Groups of a tile: as many as the fullest CTA gets through soonest (lane s - 1 looks at s).  A tile of few groups is not
       faster than its products, 0.15 to 0.27 us a step: as the weights of 1.6 to 2.8 groups, and half as large ones of DOWN. */
    const uint32_t rows = DOWN ? a.hidden : a.inter, groups = (rows + kGroup - 1) / kGroup, passes = plan.passes;
    const uint32_t s = (uint32_t)lane % kGroups + 1, most = (passes * ((groups + s - 1) / s) + gridDim.x - 1) / gridDim.x;
    const uint32_t cost = most * max(10 * s, S::parts * (12 + ta.columns / 4));
    const uint32_t size = kGroups - __reduce_min_sync(0xFFFFFFFFu, cost << 3 | (kGroups - s)) % kGroups;       /* the larger one of equals */
    const uint32_t per_pass = (groups + size - 1) / size, total = passes * per_pass;
    const uint32_t begin = (uint32_t)((unsigned long long)total * blockIdx.x / gridDim.x), end = (uint32_t)((unsigned long long)total * (blockIdx.x + 1) / gridDim.x);
    const uint32_t bytes = (DOWN ? a.inter : a.hidden) * 2, steps = (bytes + kSpan - 1) / kSpan;
    /* a stage has room for a tile's rows; the products read 128 rows all the same, those of no tile for nothing */
    const uint32_t half_bytes = size * kGroup * kSpan, weight_bytes = S::halves * half_bytes, stage_bytes = weight_bytes + S::parts * ta.columns * kSpan;
    const uint32_t stages = min((uint32_t)kMaxRing, (kRing - kRows * kSpan) / stage_bytes);
    bool fine = true, more = true;                                  /* fine: no wait of this warp has run out; more: it goes on */
    const uint32_t polls = ta.polls;
    auto for_tiles = [&](auto &&body) {
        for (uint32_t i = begin; i < end && more; ++i) {
            const uint32_t pass = i / per_pass, g0 = i % per_pass * size;
            int lo = 0, hi = active - 1;                            /* the last expert with no more passes before it */
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (s_passes[mid] <= pass) lo = mid; else hi = mid - 1;
            }
            TileAt t;
            t.expert = s_list[lo];
            t.first = s_first[lo] + (pass - s_passes[lo]) * ta.columns;
            t.n = min(ta.columns, s_first[lo + 1] - t.first);
            t.row = g0 * kGroup;
            t.count = min(size * kGroup, rows - t.row);
            body(t);
        }
    };
    uint32_t issued = 0;                                            /* steps whose weights warp 0 asked for */
    uint32_t stage = 0, phase = 0;                                  /* of this warp's next step; phase: how often the ring went round, mod 2 */
    auto step_on = [&] { if (++stage == stages) { stage = 0; phase ^= 1; } };

    if (warp == 0) {
        /* weights are nobody's output: the ring is filled with them before the kernel in front of this one has ended */
        const uint32_t leader = elect_leader();
        for_tiles([&](const TileAt &t) {
            const uint32_t row = DOWN ? t.expert * a.hidden + t.row : t.expert * 2 * a.inter + t.row, boxes = (t.count + kGroup - 1) / kGroup;
            for (uint32_t s = 0; s < steps; ++s) {
                const uint32_t bar = shared_at(&s_full[stage]), to = shared_at(smem) + stage * stage_bytes;
                if (DOWN && issued == stages) grid_wait();          /* from here on a wait goes by this kernel's own pace */
                if (!bar_wait<true>(shared_at(&s_empty[stage]), phase ^ 1, polls)) { fine = more = false; return; }
                ++issued;
                bar_arrive_and_expect(leader, bar, boxes * S::halves * kGroup * kSpan);
                uint32_t from = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!(boxes & (8u >> i))) continue;
#pragma unroll
                    for (int h = 0; h < S::halves; ++h)
                        fetch_rows(leader, to + h * half_bytes + from * kSpan, &maps.of[i], s * (kSpan / 2), row + h * a.inter + from, bar);
                    from += 128u >> i;
                }
                step_on();
            }
        });
    } else if (warp == 1) {
        const uint32_t leader = elect_leader();
        uint32_t half = 0, round = 0;                               /* of tensor memory */
        if (DOWN) grid_wait();
        for_tiles([&](const TileAt &t) {
            const uint32_t width = (t.n + 15) / 16 * 16, to = tmem + half * 128;
            const uint32_t kind = 1u << 4 | 1u << 7 | 1u << 10 | (width >> 3) << 17 | (kRows >> 4) << 24;     /* binary32 sums of bf16, K-major */
            if (!bar_wait<true>(shared_at(&s_free[half]), round ^ 1, polls)) { fine = more = false; return; }
            sums_after();
            for (uint32_t s = 0; s < steps; ++s) {
                const bool there = bar_wait<true>(shared_at(&s_full[stage]), phase, polls);
                sums_after();
                const uint32_t at = shared_at(smem) + stage * stage_bytes;
                const unsigned long long rows0 = operand(at), cols0 = operand(at + weight_bytes);
                const uint32_t quarters = (bytes - s * kSpan + 31) / 32;                                       /* of 16 elements */
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    if (k >= quarters) break;
                    product(leader, to, rows0 + 2 * k, cols0 + 2 * k, kind, s | k);
                    if (S::halves == 2) product(leader, to + 64, rows0 + (half_bytes >> 4) + 2 * k, cols0 + 2 * k, kind, s | k);
                    if (S::parts == 2) product(leader, to, rows0 + 2 * k, cols0 + (ta.columns * kSpan >> 4) + 2 * k, kind, true);
                }
                if (!there) { fine = more = false; return; }        /* asked late, beside the products: these were for nothing */
                tell_when_done(leader, shared_at(&s_empty[stage]));
                step_on();
            }
            tell_when_done(leader, shared_at(&s_sums[half]));
            half ^= 1;
            if (half == 0) round ^= 1;
        });
    } else if (warp < 4) {
        /* eight lanes per row, eight rows at a time */
        const uint32_t me = threadIdx.x - 64, r0 = me / 8, piece = me % 8;
        uint32_t pending = 0, told = 0, steps_told = 0;             /* stages filled and not told of; the next one to tell of */
        auto tell = [&] {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(shared_at(&s_full[told]));
            if (++told == stages) told = 0;
            ++steps_told;
            --pending;
        };
        if (DOWN) grid_wait();
        for_tiles([&](const TileAt &t) {
            const char *cols[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t at = t.first + min(r0 + 8 * i, t.n - 1);
                cols[i] = (DOWN ? a.h + (size_t)at * S::parts * a.h_row : a.x + s_token[at] * a.ld_x) + piece * 16;
            }
            const uint32_t place = weight_bytes + r0 * kSpan + ((piece ^ (r0 & 7)) * 16);
            for (uint32_t s = 0; s < steps; ++s) {
                const uint32_t to = shared_at(smem) + stage * stage_bytes + place, off = s * kSpan, size = off + piece * 16 < bytes ? 16u : 0u;
                if (!bar_wait(shared_at(&s_empty[stage]), phase ^ 1, polls)) { fine = more = false; return; }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (r0 + 8 * i >= t.n) break;
#pragma unroll
                    for (int p = 0; p < S::parts; ++p) copy16(to + (p * ta.columns + 8 * i) * kSpan, cols[i] + (size ? off : 0u) + p * a.h_row, size);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                step_on();
                if (++pending > kLag) {
                    asm volatile("cp.async.wait_group %0;" :: "n"(kLag) : "memory");
                    tell();
                }
            }
        });
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        while (pending) tell();
        if (lane == 0) s_told[warp - 2] = steps_told;
    } else {
        /* a thread has a row, its warp the first or the second half of the columns */
        const uint32_t row = (warp % 4) * 32 + lane, which = warp >= 8;
        float *const weights = s_weight[warp - 4];
        uint32_t half = 0, round = 0;
        if (DOWN) grid_wait();                                      /* what is written was read by kernels in front of this one */
        for_tiles([&](const TileAt &t) {
            const uint32_t width = (t.n + 15) / 16 * 8, c0 = which * width, n = t.n > c0 ? min(t.n - c0, width) : 0u;
            const uint32_t from = tmem + half * 128 + ((uint32_t)(warp % 4) << 21) + c0;
            if (!DOWN) weights[lane] = (uint32_t)lane < n ? weight_of(a, s_token[t.first + c0 + lane], (int)t.expert) : 0.0f;
            fine = fine && bar_wait(shared_at(&s_sums[half]), round, polls);
            __syncwarp();
            sums_after();
            if ((uint32_t)(warp % 4) * 32 < t.count) {              /* rows of this warp: the same for all its lanes */
                const bool in = row < t.count;
                const float right = fine ? 1.0f : NAN;              /* a wait that ran out shows */
                char *h = a.h + (t.first + c0) * (size_t)(2 * a.h_row) + (t.row + row) * 2;
                float *y = a.y + (t.first + c0) * (size_t)a.hidden + t.row + row;
                for (uint32_t c = 0; c < n; c += 8) {
                    uint32_t v[8], u[8];
                    read_sums(v, from + c);
                    if (!DOWN) read_sums(u, from + 64 + c);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (c + k >= n) break;
                        float x = __uint_as_float(v[k]);
                        if constexpr (DOWN) {
                            if (in) *y = x * right;
                            y += a.hidden;
                        } else {
                            x = weights[c + k] * right * (activate_fast(x, a.activation) * __uint_as_float(u[k]));
                            const uint16_t hi = narrow<SIFAR_BF16>(x);
                            if (in) {
                                *reinterpret_cast<uint16_t *>(h) = hi;
                                *reinterpret_cast<uint16_t *>(h + a.h_row) = narrow<SIFAR_BF16>(x - widen<SIFAR_BF16>(hi));
                            }
                            h += 2 * a.h_row;
                        }
                    }
                }
            }
            sums_before();
            __syncwarp();
            if (lane == 0 && fine) bar_arrive(shared_at(&s_free[half]));
            half ^= 1;
            if (half == 0) round ^= 1;
        });
    }
    __syncwarp();
    sums_before();
    if (__syncthreads_or(!fine)) {
        /* A wait ran out.  Nothing may be under way when the CTA ends: not the products, nor the weights, whose barriers wait
           for the gatherers that stopped, too. */
        if (warp == 0) {
            for (uint32_t i = issued > stages ? issued - stages : 0u; i < issued; ++i) {
                const uint32_t bar = shared_at(&s_full[i % stages]);
                if (lane < kGatherers / 32 && s_told[lane] <= i) bar_arrive(bar);
                __syncwarp();
                bar_wait(bar, (i / stages) & 1, kPolls);
            }
        } else if (warp == 1) {
            tell_when_done(elect_leader(), shared_at(&s_done));
            bar_wait(shared_at(&s_done), 0, kPolls);
        }
        __syncthreads();
    }
    if (warp == 1) {
        sums_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(256u));
    }
}

/* ------------------------------------------------------------------------ */
/* host                                                                      */
/* ------------------------------------------------------------------------ */
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static uint32_t polls_of_a_wait()
{
    static const uint32_t n = [] {
        const char *s = getenv("SIFAR_EXPERTS_POLLS");
        return s ? (uint32_t)strtoul(s, nullptr, 10) : kPolls;
    }();
    return n;
}

/* The driver's function by its name: the library does not link against the driver. */
static EncodeTiled encode_tiled()
{
    static const EncodeTiled f = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return (EncodeTiled)p;
    }();
    return f;
}

/* `rows` rows of `cols` bf16 elements. */
static cudaError_t map_rows(RowMaps &maps, const void *p, size_t rows, size_t cols, size_t ld_bytes)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t size[2] = {cols, rows}, stride[1] = {ld_bytes};
    for (int i = 0; i < 4; ++i) {
        const cuuint32_t box[2] = {kSpan / 2, 128u >> i}, each[2] = {1, 1};
        if (encode(&maps.of[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(p), size, stride, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    return cudaSuccess;
}

template <bool DOWN> static cudaError_t launch_tiles(cudaStream_t stream, TilesArgs t)
{
    const ExpertsArgs &a = t.e;
    RowMaps maps;
    const cudaError_t bad = DOWN ? map_rows(maps, a.down, (size_t)a.experts * a.hidden, a.inter, a.ld_down)
                                 : map_rows(maps, a.gate_up, (size_t)a.experts * 2 * a.inter, a.hidden, a.ld_gate_up);
    if (bad) return bad;
    if (cudaError_t e = cudaFuncSetAttribute(k_expert_tiles<DOWN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing)) return e;
    return launch_op(k_expert_tiles<DOWN>, dim3(kSms), dim3(kTileThreads), 1, kRing, stream, maps, t);
}

cudaError_t launch_expert_tiles(cudaStream_t stream, const ExpertsArgs &a)
{
    TilesArgs t;
    t.e = a;
    /* columns of a pass: four times an expert's share of the choices, were they spread evenly; more take another pass */
    const uint32_t most = 4 * ((a.tokens * a.top_k + a.experts - 1) / a.experts), need = most < a.tokens ? most : a.tokens;
    t.columns = need <= 16 ? 16 : need <= 32 ? 32 : 64;
    t.polls = polls_of_a_wait();
    if (cudaError_t e = launch_tiles<false>(stream, t)) return e;
    return launch_tiles<true>(stream, t);
}

}  /* namespace sifar */
