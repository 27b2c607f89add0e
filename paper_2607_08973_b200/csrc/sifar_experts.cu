/*
 * sifar_experts.cu - the chosen experts' products for a few tokens: one rank's partial of the next all-reduce.
 *
 * Every chosen expert's weights go once from memory through registers into matrix instructions, and that is what bounds
 * the call: a token has 2 operations per weight, the memory takes 2 bytes for one.  So the weights are the 16 rows of
 * an instruction and the tokens its 8 columns.  A lane loads 16 bytes in a row of a weight row; the products' order
 * over k is free, so the eight elements become two instructions' fragments as they lie, with the tokens' taken from the same
 * places.  No weight passes through shared memory.
 *
 *   k_up_few, k_down_few     up to 8 tokens; up to 16 or 32 where sifar_experts_tiles.cu does not take them.  All tokens are columns for
 *                            every expert, the warps of a CTA share the rows' length.
 *   k_products<UP / DOWN>    more of those: an expert's tokens are gathered to columns, each warp has 16 rows of its own.
 *   k_align                  ... the tokens' rows for those and for the tiles, on whole pieces.
 *   k_gather                 ... and the sum over a token's choices, in their order.
 *
 * bf16: what goes into the second product is kept as two bf16 values, the rounded one and what it leaves (16 bits).  binary32 values are
 * three bf16 ones, six instructions for one: as fused multiply-adds the same work was bound by loads from shared memory (83 tokens,
 * 8 experts of 625 x 1216: 239 us, 132 now; 31 tokens, 64 experts of 1000 x 512: 199, 104).
 *
 * One bf16 token with 8 of 128 experts of 768 x 4096 takes 32.6 us, 4.6 TB/s (151 MB): two starts, in which the lists are made and
 * the first weights come; the second kernel's CTAs find room when the first one's end.  13 binary32 tokens, 7 experts of 333 x 1001 whose rows
 * start anywhere: 33.6 us for 28 MB, bound by the starts and by instructions, shuffles that put rows together among them.
 */
#include "sifar_experts.cuh"
#include "sifar_experts_shape.cuh"

namespace sifar {

constexpr int kWarps = kExpertWarps, kThreads = kExpertThreads;
constexpr int kBlock = 64;                   /* bytes of a row that the four lanes of a row load at once */
constexpr int kAhead = 4;                    /* blocks that a lane loads together: 256 bytes of a row */
constexpr uint32_t kFetchAhead = 6;          /* items of a warp that k_down_few asks for before its values are there */
constexpr int kFew = 8, kFewMost = 32;       /* tokens that fit one instruction's columns, four ones' */
constexpr int kChunk = 512;                  /* bytes of the weights' rows that go with what is in shared memory at a time (more tokens) */

/* ------------------------------------------------------------------------ */
/* loads                                                                     */
/* ------------------------------------------------------------------------ */
/* Plain ones: a kernel may have been started while the one in front still wrote what it reads, so nothing is constant for its life. */
__device__ __forceinline__ uint4 load_once(const char *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

/*
 * What a lane has on the way of its two rows: 16 bytes of each of kAhead blocks, a block being the 64 bytes of the row's four lanes.
 * Rows that start anywhere (not VEC) are loaded as the aligned vectors that hold them, and put together when they are used: the
 * vector behind a lane's own is the next lane's, the last lane's the first one's of the next block, of which the first lane has
 * one more.
 */
template <bool VEC> struct Weights {
    static constexpr int n = VEC ? kAhead : kAhead + 1;
    uint4 a[n], b[n];
    uint32_t sh_a, sh_b;

    static __device__ __forceinline__ uint32_t row(uint4 (&v)[n], const char *p, uint32_t at, uint32_t bytes)
    {
        const uint32_t sh = VEC ? 0u : (uint32_t)(uintptr_t)p & 15u;
        const char *const from = p - sh + at;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            v[i] = make_uint4(0u, 0u, 0u, 0u);
            if (p && at + i * kBlock < bytes + sh && (i < kAhead || (threadIdx.x & 3) == 0)) {
                if (VEC) v[i] = load_once(from + i * kBlock);
                else v[i] = *reinterpret_cast<const uint4 *>(from + i * kBlock);
            }
        }
        return sh;
    }
    /* From byte `at` (the lane's own) of two rows of `bytes`; a row may be missing. */
    __device__ __forceinline__ void load(const char *ra, const char *rb, uint32_t at, uint32_t bytes)
    {
        sh_a = row(a, ra, at, bytes);
        sh_b = row(b, rb, at, bytes);
    }
    static __device__ __forceinline__ uint4 use(const uint4 (&v)[n], uint32_t sh, int i, int left)
    {
        if (VEC) return v[i];
        const int lane = threadIdx.x & 31, from = (lane & ~3) | ((lane + 1) & 3);
        const bool first = (lane & 3) == 0;
        const uint4 own = v[i], behind = v[i + 1 < n ? i + 1 : i];
        const uint4 give = make_uint4(first ? behind.x : own.x, first ? behind.y : own.y, first ? behind.z : own.z, first ? behind.w : own.w);
        uint4 hi;
        hi.x = __shfl_sync(0xFFFFFFFFu, give.x, from); hi.y = __shfl_sync(0xFFFFFFFFu, give.y, from);
        hi.z = __shfl_sync(0xFFFFFFFFu, give.z, from); hi.w = __shfl_sync(0xFFFFFFFFu, give.w, from);
        return shifted(own, hi, sh, left);
    }
    /* Block i; `left`: bytes of the rows from the lane's own on.  All lanes together. */
    __device__ __forceinline__ uint4 of_a(int i, int left) const { return use(a, sh_a, i, left); }
    __device__ __forceinline__ uint4 of_b(int i, int left) const { return use(b, sh_b, i, left); }
};

/* An asynchronous copy of 4 bytes into shared memory; of 0 bytes: zeros. */
__device__ __forceinline__ void copy4(void *to, const char *from, uint32_t bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
/* ... of 16 bytes. */
__device__ __forceinline__ void copy16(void *to, const char *from, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ void multiply(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
/*
 * binary32: a value is the sum of three bf16 ones, each the nearest to what the ones before it leave (24 bits).  Of the nine products
 * of two values' parts the three least are left out, together 2^-25 of the product.  Values that are not finite, or that round
 * to no finite bf16 value, give NaN.
 */
struct Parts { uint2 high, mid, low; };
__device__ __forceinline__ uint32_t bf16_pair(float first, float second)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(second), "f"(first));
    return r;
}
__device__ __forceinline__ void part(uint32_t first, uint32_t second, uint32_t &high, uint32_t &mid, uint32_t &low)
{
    float a = __uint_as_float(first), b = __uint_as_float(second);
    high = bf16_pair(a, b);
    a -= __uint_as_float(high << 16); b -= __uint_as_float(high & 0xFFFF0000u);
    mid = bf16_pair(a, b);
    a -= __uint_as_float(mid << 16); b -= __uint_as_float(mid & 0xFFFF0000u);
    low = bf16_pair(a, b);
}
__device__ __forceinline__ Parts parts_of(const uint4 &v)
{
    Parts p;
    part(v.x, v.y, p.high.x, p.mid.x, p.low.x);
    part(v.z, v.w, p.high.y, p.mid.y, p.low.y);
    return p;
}
/* A block's weights as the instructions take them. */
template <int DT> __device__ __forceinline__ auto operand(const uint4 &v)
{
    if constexpr (DT == SIFAR_BF16) return v;
    else return parts_of(v);
}

/*
 * One block of 16 weight rows (a lane's rows g and g + 8) with 8 N tokens (the lane's: g, g + 8, ...).  An instruction waits for the one
 * before it with the same sums: those of the N groups take turns.
 */
template <int N> __device__ __forceinline__ void multiply_block(float (*c)[4], const uint4 &a, const uint4 &b, const uint4 (&x)[N])
{
#pragma unroll
    for (int q = 0; q < N; ++q) multiply(c[q], a.x, b.x, a.y, b.y, x[q].x, x[q].y);
#pragma unroll
    for (int q = 0; q < N; ++q) multiply(c[q], a.z, b.z, a.w, b.w, x[q].z, x[q].w);
}
/* The instructions cut their sums off, so the large products have sums of their own, and both kinds are taken over by rounded adds after
   at most eight blocks (40 tokens of 16384 columns: off by 6.6e-7 of the largest value, with a row in one sum 4.0e-5, a plain binary32
   product 9.9e-7; 83 tokens, 8 experts of 625 x 1216: 4.0e-7, 3.1e-6, for 132 us in place of 127). */
template <int N> __device__ __forceinline__ void multiply_block(float (*c)[4], float (*less)[4], const Parts &a, const Parts &b, const Parts (&x)[N])
{
    const auto all = [&](float (*to)[4], const uint2 &a0, const uint2 &b0, uint2 Parts::*of) {
#pragma unroll
        for (int q = 0; q < N; ++q) multiply(to[q], a0.x, b0.x, a0.y, b0.y, (x[q].*of).x, (x[q].*of).y);
    };
    all(less, a.low, b.low, &Parts::high);
    all(less, a.high, b.high, &Parts::low);
    all(less, a.mid, b.mid, &Parts::mid);
    all(less, a.mid, b.mid, &Parts::high);
    all(less, a.high, b.high, &Parts::mid);
    all(c, a.high, b.high, &Parts::high);
}

/* ------------------------------------------------------------------------ */
/* up to 8 G tokens                                                          */
/* ------------------------------------------------------------------------ */
/* A lane's accumulators for 16 rows x 8 G tokens. */
template <int DT, int G> struct Few {
    float c[G][4] = {}, less[DT == SIFAR_F32 ? G : 1][4] = {};
    __device__ __forceinline__ void join()                         /* c: all of it */
    {
        if constexpr (DT == SIFAR_F32) {
#pragma unroll
            for (int q = 0; q < G; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) c[q][i] += less[q][i];
        }
    }
    static __device__ __forceinline__ void store(float *red, const float (&v)[G][4])   /* red: 16 rows x 8 G tokens */
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
#pragma unroll
        for (int q = 0; q < G; ++q) {
            *reinterpret_cast<float2 *>(red + g * 8 * G + q * 8 + 2 * j) = make_float2(v[q][0], v[q][1]);
            *reinterpret_cast<float2 *>(red + (g + 8) * 8 * G + q * 8 + 2 * j) = make_float2(v[q][2], v[q][3]);
        }
    }
    /* Adds the columns whose bit is set. */
    __device__ __forceinline__ void add_to(float (&sum)[G][4], uint32_t columns = 0xFFFFFFFFu)
    {
        columns >>= 2 * (threadIdx.x & 3);
        join();
#pragma unroll
        for (int q = 0; q < G; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[q][i] += columns >> (8 * q + (i & 1)) & 1u ? c[q][i] : 0.0f;
    }
};

/* The experts that have tokens, in their order, and which (bit t: token t).  Returns how many. */
__device__ __forceinline__ int list_few(const ExpertsArgs &a, uint16_t *list, uint32_t *tokens, uint32_t *bits, int *scratch)
{
    for (uint32_t e = threadIdx.x; e < a.experts; e += kThreads) bits[e] = 0u;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < a.tokens * a.top_k; i += kThreads) {
        const uint32_t e = local_expert(a, a.indices[i]);
        if (e < a.experts) atomicOr(&bits[e], 1u << (i / a.top_k));
    }
    __syncthreads();
    return keep_in_order(a.experts, scratch, [&](uint32_t e) { return bits[e] != 0u; },
                         [&](int at, uint32_t e) { list[at] = (uint16_t)e; tokens[at] = bits[e]; });
}

/*
 * All experts' rows lie in a row and every CTA has an equal share of it, 8 gate rows and the 8 up rows that go with them at a
 * time, so a product's gate and up lie 8 rows apart.  The warps take the rows' 256-byte pieces in turn, in groups with tiles of their
 * own where rows have fewer than eight; the next pieces are under way while these are multiplied, across tiles too.
 */
template <int DT, int G, bool VEC, bool XVEC>
__global__ void __launch_bounds__(kThreads, kFewCtas<G>) k_up_few(const __grid_constant__ ExpertsArgs a)
{
    constexpr int es = DT == SIFAR_BF16 ? 2 : 4;
    extern __shared__ __align__(128) char smem[];                   /* tokens x x_row */
    __shared__ uint32_t s_bits[SIFAR_ROUTE_MAX_EXPERTS], s_tokens[SIFAR_ROUTE_MAX_EXPERTS];
    __shared__ uint16_t s_list[SIFAR_ROUTE_MAX_EXPERTS];
    __shared__ int s_scratch[kWarps];
    __shared__ __align__(16) float s_red[2][kWarps][16 * 8 * G];
    static_assert(sizeof s_bits + sizeof s_tokens + sizeof s_list + sizeof s_scratch + sizeof s_red <= kFewStatic<G>, "what few_ctas() counts");
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, g = lane >> 2, j = lane & 3;
    grid_wait();
    grid_let_next_in();
    const uint32_t bytes = a.hidden * es, per_row = a.x_row / 16, all = a.tokens * per_row;
    /* the tokens' rows, zeros behind their ends: on their way while the experts are listed */
    constexpr bool kCopy = XVEC || DT == SIFAR_F32;
    if (XVEC) {
        for (uint32_t i = threadIdx.x; i < all; i += kThreads) {
            const uint32_t t = i / per_row, at = (i - t * per_row) * 16;
            copy16(smem + i * 16, at < bytes ? a.x + t * a.ld_x + at : a.x, at < bytes ? 16u : 0u);
        }
    } else if (kCopy) {
        for (uint32_t t = 0; t < a.tokens; ++t)
#pragma unroll 4
            for (uint32_t at = threadIdx.x * 4; at < a.x_row; at += kThreads * 4)
                copy4(smem + t * a.x_row + at, at < bytes ? a.x + t * a.ld_x + at : a.x, at < bytes ? 4u : 0u);
    }
    if (kCopy) copies_commit();
    const uint32_t pairs = (uint32_t)list_few(a, s_list, s_tokens, s_bits, s_scratch) * a.inter;
    const uint32_t begin = (uint32_t)((unsigned long long)pairs * blockIdx.x / gridDim.x), end = (uint32_t)((unsigned long long)pairs * (blockIdx.x + 1) / gridDim.x);
    constexpr uint32_t kPiece = kAhead * kBlock;
    const uint32_t pieces = (bytes + kPiece - 1) / kPiece;
    const uint32_t group = pieces <= 1 ? 1u : pieces <= 2 ? 2u : pieces <= 4 ? 4u : (uint32_t)kWarps, tiles = kWarps / group;     /* warps of a tile, tiles at a time */
    const uint32_t steps = (pieces + group - 1) / group, span = group * kPiece;
    auto rows_of = [&](uint32_t p, const char *&ra, const char *&rb) {
        ra = rb = nullptr;
        p += warp / group * 8 + g;
        if (p >= end) return;
        const uint32_t which = p / a.inter;
        ra = a.gate_up + ((unsigned long long)s_list[which] * 2 * a.inter + (p - which * a.inter)) * a.ld_gate_up;
        rb = ra + (unsigned long long)a.inter * a.ld_gate_up;
    };
    const uint32_t mine = warp % group * kPiece + j * 16;
    const char *ra, *rb;
    rows_of(begin, ra, rb);
    Weights<VEC> next;
    next.load(ra, rb, mine, bytes);

    if (kCopy) {
        copies_wait<0>();
    } else {
        for (uint32_t i0 = threadIdx.x; i0 < all; i0 += 4 * kThreads) {
            uint4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t i = i0 + k * kThreads, t = i / per_row, at = (i - t * per_row) * 16;
                v[k] = i < all && at < bytes ? load_shifted(a.x + t * a.ld_x + at, bytes - at) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i0 + k * kThreads < all) *reinterpret_cast<uint4 *>(smem + (i0 + k * kThreads) * 16) = v[k];
        }
    }
    __syncthreads();

    int parity = 0;
    for (uint32_t p = begin; p < end; p += 8 * tiles, parity ^= 1) {
        Few<DT, G> acc;
        float sum[G][4] = {};
        for (uint32_t s = 0; s < steps; ++s) {
            const Weights<VEC> now = next;
            const uint32_t at = s * span + mine;
            if (s + 1 < steps) {
                next.load(ra, rb, at + span, bytes);
            } else {
                rows_of(p + 8 * tiles, ra, rb);
                next.load(ra, rb, mine, bytes);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (at - j * 16 + i * kBlock >= bytes) break;       /* the same for all lanes */
                const int left = (int)bytes - (int)(at + i * kBlock);
                const auto wa = operand<DT>(now.of_a(i, left)), wb = operand<DT>(now.of_b(i, left));
                uint4 x[G];
#pragma unroll
                for (int q = 0; q < G; ++q) {
                    x[q] = make_uint4(0u, 0u, 0u, 0u);
                    if ((uint32_t)(q * 8 + g) < a.tokens) x[q] = *reinterpret_cast<const uint4 *>(smem + (q * 8 + g) * a.x_row + at + i * kBlock);
                }
                if constexpr (DT == SIFAR_BF16) {
                    multiply_block<G>(acc.c, wa, wb, x);
                } else {
                    Parts parts[G];
#pragma unroll
                    for (int q = 0; q < G; ++q) parts[q] = parts_of(x[q]);
                    multiply_block<G>(acc.c, acc.less, wa, wb, parts);
                }
            }
            if constexpr (DT == SIFAR_F32) {                        /* a piece's sums */
                acc.add_to(sum);
                acc = Few<DT, G>();
            }
        }
        Few<DT, G>::store(s_red[parity][warp], DT == SIFAR_F32 ? sum : acc.c);
        __syncthreads();                                            /* the other parity's sums are read by now */
        /* a warp has a pair of each tile, its lanes the tokens */
        const uint32_t t = lane;
        for (uint32_t tile = 0; tile < tiles; ++tile) {
            const uint32_t pair = p + tile * 8 + warp, which = pair / a.inter;
            if (pair >= end) break;
            if (t >= a.tokens || !(s_tokens[which] >> t & 1u)) continue;
            float gate = 0.0f, up = 0.0f;
            for (uint32_t w = tile * group; w < (tile + 1) * group; ++w) { gate += s_red[parity][w][warp * 8 * G + t]; up += s_red[parity][w][(warp + 8) * 8 * G + t]; }
            const size_t low = (size_t)a.tokens * a.h_row;
            store_h<DT == SIFAR_BF16 ? 2 : 0>(a, a.h + which * (DT == SIFAR_BF16 ? 2 : 1) * low + t * (size_t)a.h_row, low, pair - which * a.inter,
                        weight_of(a, t, s_list[which]) * (activate(gate, a.activation) * up));
        }
    }
}

/* What an item's values take: 256 bytes of each row, eight of which are read at once, shifted by half of the banks.
   0: too much for two items of each warp, the values are read where they are used. */
template <int DT, int G> struct Staged {
    static constexpr int row = kAhead * kBlock + 64, bytes = DT == SIFAR_F32 ? 8 * G * row : G == 1 ? 2 * 8 * row : 0;
};
constexpr int kMaxSplit = 8;                 /* CTAs that share columns of the output */

/* Into the same place of CTA `rank`'s shared memory. */
__device__ __forceinline__ void store_cluster(float *local, uint32_t rank, float v)
{
    asm volatile("{\n\t.reg .u32 q;\n\tmapa.shared::cluster.u32 q, %0, %1;\n\tst.shared::cluster.f32 [q], %2;\n\t}"
                 :: "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(rank), "f"(v) : "memory");
}

/*
 * A CTA has an equal share of the output's columns, 16 at a time, and goes over all experts that have tokens; its warps take
 * the 256-byte pieces of the experts' rows in turn.  Where there are few columns, the CTAs of a cluster share them and take turns, and
 * the first one adds their sums up.  Tokens that did not choose an expert have zeros there and are not read; an item's products are added
 * to the tokens that chose its expert alone, since zero times what its weights may hold need not be zero.
 * HALF (bf16, up to 4 tokens): both parts of the products' values are columns of one instruction.
 */
template <int DT, int G, bool VEC, bool HALF>
__global__ void __launch_bounds__(kThreads, kFewCtas<G>) k_down_few(const __grid_constant__ ExpertsArgs a)
{
    constexpr int es = DT == SIFAR_BF16 ? 2 : 4;
    __shared__ uint32_t s_bits[SIFAR_ROUTE_MAX_EXPERTS], s_tokens[SIFAR_ROUTE_MAX_EXPERTS];
    __shared__ uint16_t s_list[SIFAR_ROUTE_MAX_EXPERTS];
    __shared__ int s_scratch[kWarps];
    __shared__ __align__(16) float s_red[kWarps][16 * 8 * G], s_part[kMaxSplit][16 * 8 * G];
    extern __shared__ __align__(128) char smem[];                   /* not HALF: each warp's two items' values */
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, g = lane >> 2, j = lane & 3;
    if (a.split > 1) cluster_arrive();                              /* a CTA's shared memory may be written once it has started */
    /* the choices were complete before the kernel in front of this one let it in, so they may be read before it ends */
    const int active = list_few(a, s_list, s_tokens, s_bits, s_scratch);
    const uint32_t bytes = a.inter * es, pieces = (bytes + kAhead * kBlock - 1) / (kAhead * kBlock), items = (uint32_t)active * pieces;
    const uint32_t split = a.split, rank = split > 1 ? cluster_rank() : 0u, block = blockIdx.x / split, blocks = gridDim.x / split;
    const uint32_t begin = (uint32_t)((unsigned long long)a.hidden * block / blocks), end = (uint32_t)((unsigned long long)a.hidden * (block + 1) / blocks);
    const uint32_t warp0 = rank * kWarps + warp, turn = split * kWarps;                  /* the warp's first item, and how many lie between two */
    auto load = [&](Weights<VEC> &w, uint32_t col, uint32_t item) {
        const char *ra = nullptr, *rb = nullptr;
        if (item < items) {
            const unsigned long long row = (unsigned long long)s_list[item / pieces] * a.hidden + col + g;
            if (col + g < end) ra = a.down + row * a.ld_down;
            if (col + g + 8 < end) rb = a.down + (row + 8) * a.ld_down;
        }
        w.load(ra, rb, item % pieces * (kAhead * kBlock) + j * 16, bytes);
    };
    Weights<VEC> next;
    load(next, begin, warp0);
    /* the next items' weights, too, as far as the L2: a lane has half a row's piece of each */
    for (uint32_t k = 1; k <= kFetchAhead; ++k) {
        const uint32_t item = warp0 + k * turn, c = begin + lane / 2, at = item % pieces * (kAhead * kBlock) + (lane & 1) * 128;
        if (item >= items) break;
        if (c < end && at < bytes)
            asm volatile("prefetch.global.L2 [%0];" :: "l"(a.down + ((unsigned long long)s_list[item / pieces] * a.hidden + c) * a.ld_down + at));
    }
    grid_wait();
    grid_let_next_in();
    if (split > 1) cluster_wait();
    const size_t low = (size_t)a.tokens * a.h_row;
    /* the values that go with an item, two rows at a time (bf16: a token's parts, the second ones 8 G rows on), zeros behind their ends */
    constexpr bool kStaged = !HALF && Staged<DT, G>::bytes > 0;
    char *const staged = smem + warp * (2 * Staged<DT, G>::bytes);
    auto fetch = [&](uint32_t item, int half) {
        if (item < items) {
            const uint32_t which = item / pieces, at = item % pieces * (kAhead * kBlock) + (lane & 15) * 16, size = at < a.h_row ? 16u : 0u;
            const char *const h = a.h + (size_t)which * (DT == SIFAR_BF16 ? 2 : 1) * low + (size ? at : 0u);
            char *const to = staged + half * Staged<DT, G>::bytes + (lane & 15) * 16;
            uint32_t rest = s_tokens[which];
            while (rest) {
                uint32_t t = __ffs(rest) - 1;
                rest &= rest - 1u;
                if constexpr (DT == SIFAR_BF16) {
                    const uint32_t part = lane / 16;
                    copy16(to + (part * 8 * G + t) * Staged<DT, G>::row, h + part * low + t * (size_t)a.h_row, size);
                } else {
                    if (lane >= 16 && rest) t = __ffs(rest) - 1;
                    rest &= rest - 1u;
                    copy16(to + t * Staged<DT, G>::row, h + t * (size_t)a.h_row, size);
                }
            }
        }
        copies_commit();
    };
    for (uint32_t col = begin; col < end; col += 16) {
        float sum[G][4] = {};
        int half = 0;
        if (kStaged) fetch(warp0, 0);
        for (uint32_t item = warp0; item < items; item += turn, half ^= 1) {
            Few<DT, G> acc;
            const Weights<VEC> now = next;
            const uint32_t which = item / pieces, at = item % pieces * (kAhead * kBlock) + j * 16, tokens = s_tokens[which];
            const bool more = item + turn < items;
            if constexpr (HALF) {
                uint4 x[kAhead];
                const uint32_t t = g & 3;
                const char *const from = a.h + (size_t)which * 2 * low + t * (size_t)a.h_row + (g >= 4 ? low : 0) + at;
#pragma unroll
                for (int i = 0; i < kAhead; ++i)                    /* rows of h are filled up with zeros to 16 bytes */
                    x[i] = (tokens >> t & 1u) && at + i * kBlock < a.h_row ? __ldcg(reinterpret_cast<const uint4 *>(from + i * kBlock)) : make_uint4(0u, 0u, 0u, 0u);
                load(next, more ? col : col + 16, more ? item + turn : warp0);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (at - j * 16 + i * kBlock >= bytes) break;
                    const int left = (int)bytes - (int)(at + i * kBlock);
                    multiply_block<1>(acc.c, now.of_a(i, left), now.of_b(i, left), {x[i]});
                }
                acc.add_to(sum, tokens | tokens << 4);
            } else {
                load(next, more ? col : col + 16, more ? item + turn : warp0);
                if (kStaged) fetch(item + turn, half ^ 1);
                uint4 wa[kAhead], wb[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int left = (int)bytes - (int)(at + i * kBlock);
                    wa[i] = now.of_a(i, left);
                    wb[i] = now.of_b(i, left);
                }
                if (kStaged) copies_wait<1>();
                __syncwarp();
                const char *const x0 = staged + half * Staged<DT, G>::bytes + j * 16;
                constexpr bool two = DT == SIFAR_BF16;
                constexpr int N = G < 2 ? 1 : 2;                    /* groups at a time */
#pragma unroll
                for (int q = 0; q < G; q += N) {
                    if (!(tokens >> (8 * q) & (N == 2 ? 0xFFFFu : 0xFFu))) continue;
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        uint4 x[N], y[N];
#pragma unroll
                        for (int k = 0; k < N; ++k) {
                            const uint32_t t = (q + k) * 8 + g;
                            const char *const from = a.h + (size_t)which * (two ? 2 : 1) * low + t * (size_t)a.h_row + at + i * kBlock;
                            x[k] = y[k] = make_uint4(0u, 0u, 0u, 0u);
                            if (!(tokens >> t & 1u)) continue;
                            if (kStaged) {
                                x[k] = *reinterpret_cast<const uint4 *>(x0 + t * Staged<DT, G>::row + i * kBlock);
                                if (two) y[k] = *reinterpret_cast<const uint4 *>(x0 + (t + 8 * G) * Staged<DT, G>::row + i * kBlock);
                            } else if (at + i * kBlock < a.h_row) {
                                x[k] = __ldcg(reinterpret_cast<const uint4 *>(from));
                                if (two) y[k] = __ldcg(reinterpret_cast<const uint4 *>(from + low));
                            }
                        }
                        if constexpr (two) {
                            multiply_block<N>(acc.c + q, wa[i], wb[i], x);
                            multiply_block<N>(acc.c + q, wa[i], wb[i], y);
                        } else {
                            Parts parts[N];
#pragma unroll
                            for (int k = 0; k < N; ++k) parts[k] = parts_of(x[k]);
                            multiply_block<N>(acc.c + q, acc.less + q, parts_of(wa[i]), parts_of(wb[i]), parts);
                        }
                    }
                }
                acc.add_to(sum, tokens);
                __syncwarp();
            }
        }
        if (kStaged) copies_wait<0>();
        Few<DT, G>::store(s_red[warp], sum);
        __syncthreads();
        auto out = [&](uint32_t t, uint32_t r, float v) { reinterpret_cast<typename Elem<DT>::type *>(a.out + t * a.ld_out)[col + r] = narrow<DT>(v); };
        for (uint32_t i = threadIdx.x; i < 16 * a.tokens; i += kThreads) {
            const uint32_t r = i % 16, t = i / 16;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) v += s_red[w][r * 8 * G + t];
            if (HALF) {
                float rest = 0.0f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) rest += s_red[w][r * 8 * G + t + 4];
                v += rest;
            }
            if (split > 1) store_cluster(&s_part[rank][i], 0, v);
            else if (col + r < end) out(t, r, v);
        }
        if (split > 1) {
            cluster_arrive();
            cluster_wait();
            if (rank == 0)
                for (uint32_t i = threadIdx.x; i < 16 * a.tokens; i += kThreads) {
                    float v = 0.0f;
                    for (uint32_t k = 0; k < split; ++k) v += s_part[k][i];
                    if (col + i % 16 < end) out(i / 16, i % 16, v);
                }
            if (col + 16 < end) {                                   /* before the next columns' sums come */
                cluster_arrive();
                cluster_wait();
            }
        }
        __syncthreads();
    }
}

/* ------------------------------------------------------------------------ */
/* more tokens                                                               */
/* ------------------------------------------------------------------------ */
/*
 * Parts that the tokens' values come in, all bf16; groups of eight columns; columns of a pass.  bf16: the values of the second product
 * are two parts, in columns of their own.  binary32: three parts, one behind the other in a row.
 * In shared memory rows are shifted: eight lanes read 64 bytes of two rows, or sixteen 32 of four.
 */
template <int DT, bool DOWN> struct Pass {
    static constexpr int parts = DT == SIFAR_F32 ? 3 : DOWN ? 2 : 1;
    static constexpr int groups = DT == SIFAR_F32 ? 4 : 8;
    static constexpr int tokens = DT == SIFAR_F32 ? 32 : 64 / parts;
    static constexpr int piece = DT == SIFAR_F32 ? kChunk / 2 : kChunk;       /* bytes of a part that go with a chunk of the weights */
    static constexpr int row = DT == SIFAR_F32 ? 3 * piece + 32 : piece + 64;
    static constexpr int half = groups * 8 * row, shared = 2 * half;
};

/*
 * A unit is 128 rows of one expert with 8 up to Pass::tokens of its tokens: 64 gate and 64 up rows (UP), or 128 columns of the
 * output (DOWN).  The columns' rows come through shared memory 512 bytes at a time, the next ones under way; weights as
 * above, 256 bytes ahead.
 */
template <int DT, bool DOWN, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) k_products(const __grid_constant__ ExpertsArgs a)
{
    using P = Pass<DT, DOWN>;
    constexpr int es = DT == SIFAR_BF16 ? 2 : 4, G = P::tokens / 8;
    extern __shared__ __align__(128) char smem[];                   /* 2 x columns x Pass::row; at first each expert's tokens as bits */
    __shared__ uint16_t s_place[SIFAR_ROUTE_MAX_EXPERTS], s_list[SIFAR_ROUTE_MAX_EXPERTS], s_first[SIFAR_ROUTE_MAX_EXPERTS + 1], s_passes[SIFAR_ROUTE_MAX_EXPERTS + 1];
    __shared__ uint8_t s_token[SIFAR_EXPERTS_MAX_TOKENS * SIFAR_ROUTE_MAX_TOP_K];
    __shared__ unsigned long long s_sum[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, g = lane >> 2, j = lane & 3;
    if (!DOWN) grid_wait();
    grid_let_next_in();
    const uint32_t rows = DOWN ? a.hidden : a.inter, per = DOWN ? 128u : 64u, tiles = (rows + per - 1) / per;
    /* Columns of a pass: as many as the fullest CTA gets through soonest.  What does not depend on them takes as long as 48 columns. */
    auto pick = [&](const auto &n) {
        unsigned long long passes = 0;                              /* with 8, 16, 32, 64 columns, 16 bits each */
#pragma unroll
        for (uint32_t m : n)
#pragma unroll
            for (int i = 0; i < 4; ++i) passes += (unsigned long long)((m + (8u << i) - 1) >> (3 + i)) << (16 * i);
#pragma unroll
        for (int d = 16; d; d >>= 1) passes += __shfl_xor_sync(0xFFFFFFFFu, passes, d);
        if (lane == 0) s_sum[warp] = passes;
        __syncthreads();
        passes = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) passes += s_sum[w];
        __syncthreads();
        uint32_t best = 0xFFFFFFFFu, columns = P::tokens;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            const uint32_t cost = ((uint32_t)(passes >> (16 * i) & 0xFFFFu) * tiles + gridDim.x - 1) / gridDim.x * (48 + (8u << i));
            if ((8 << i) <= P::tokens && cost < best) { best = cost; columns = 8u << i; }
        }
        return columns;
    };
    const ExpertPlan plan = plan_experts<kThreads>(a, pick, reinterpret_cast<uint32_t *>(smem), s_sum, s_place, s_list, s_first, s_passes, s_token, !DOWN && blockIdx.x == 0);
    __syncthreads();
    const uint32_t units = plan.passes * tiles;
    const uint32_t bytes = (DOWN ? a.inter : a.hidden) * es, steps = (bytes + kChunk - 1) / kChunk;
    const uint32_t begin = (uint32_t)((unsigned long long)units * blockIdx.x / gridDim.x), end = (uint32_t)((unsigned long long)units * (blockIdx.x + 1) / gridDim.x);

    struct Unit { uint32_t expert, tile, first, n; };               /* tokens first .. first + n - 1 of the list */
    auto unit = [&](uint32_t u) {
        const uint32_t pass = u / tiles;
        int lo = 0, hi = plan.active - 1;                           /* the last expert with no more passes before it */
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (s_passes[mid] <= pass) lo = mid; else hi = mid - 1;
        }
        const uint32_t first = s_first[lo] + (pass - s_passes[lo]) * plan.columns;
        return Unit{s_list[lo], u % tiles, first, min(plan.columns, s_first[lo + 1] - first)};
    };
    auto rows_of = [&](uint32_t u, const char *&ra, const char *&rb) {
        ra = rb = nullptr;
        if (u >= end) return;
        const Unit t = unit(u);
        const unsigned long long e = t.expert;
        if (DOWN) {
            const uint32_t r = t.tile * 128 + warp * 16 + g;
            if (r < a.hidden) ra = a.down + (e * a.hidden + r) * a.ld_down;
            if (r + 8 < a.hidden) rb = a.down + (e * a.hidden + r + 8) * a.ld_down;
        } else {
            const uint32_t r = t.tile * 64 + warp * 8 + g;
            if (r >= a.inter) return;
            ra = a.gate_up + (e * 2 * a.inter + r) * a.ld_gate_up;
            rb = ra + (unsigned long long)a.inter * a.ld_gate_up;
        }
    };

    const char *ra, *rb;
    rows_of(begin, ra, rb);
    Weights<VEC> next;
    next.load(ra, rb, j * 16, bytes);
    if (DOWN) grid_wait();                                          /* what was loaded so far no kernel writes */
    /* column c: token c of the pass */
    const uint32_t part_row = DOWN ? a.h_row : ((a.hidden * 2 + 15u) & ~15u);
    auto fetch = [&](const Unit &at, uint32_t step, int buffer) {
        char *const to = smem + buffer * P::half;
        for (uint32_t i = threadIdx.x; i < at.n * P::parts * (P::piece / 16); i += kThreads) {
            const uint32_t c = i / (P::piece / 16), piece = i % (P::piece / 16) * 16, off = step * P::piece + piece;
            const uint32_t token = c / P::parts, part = c % P::parts, in_list = at.first + token, take = off < part_row ? 16u : 0u;
            const char *const row = DOWN ? a.h + ((size_t)in_list * P::parts + part) * a.h_row : a.x + s_token[in_list] * a.ld_x + part * part_row;
            char *const dst = to + (DT == SIFAR_F32 ? token * P::row + part * P::piece : (part * (G * 8) + token) * P::row) + piece;
            copy16(dst, row + (take ? off : 0u), take);
        }
        copies_commit();
    };
    Unit behind = {};
    int buffer = 0;
    if (begin < end) {
        behind = unit(begin);
        fetch(behind, 0, 0);
    }

    for (uint32_t u = begin; u < end; ++u) {
        const Unit at = behind;
        const uint32_t n = at.n, groups = (n + 7) / 8;
        if (u + 1 < end) behind = unit(u + 1);
        float acc[P::groups][4] = {}, less[DT == SIFAR_F32 ? P::groups : 1][4] = {}, sum[DT == SIFAR_F32 ? P::groups : 1][4] = {};
        for (uint32_t s = 0; s < steps; ++s, buffer ^= 1) {
            copies_wait<0>();
            __syncthreads();                                        /* this chunk is there, the one before has been read */
            if (s + 1 < steps) fetch(at, s + 1, buffer ^ 1);
            else if (u + 1 < end) fetch(behind, 0, buffer ^ 1);
            const char *const cols = smem + buffer * P::half;
#pragma unroll 1
            for (int half = 0; half < kChunk / (kAhead * kBlock); ++half) {
                const uint32_t off = s * kChunk + half * kAhead * kBlock;
                const Weights<VEC> now = next;
                if (off + kAhead * kBlock < steps * kChunk) {
                    next.load(ra, rb, off + kAhead * kBlock + j * 16, bytes);
                } else {
                    rows_of(u + 1, ra, rb);
                    next.load(ra, rb, j * 16, bytes);
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (off + i * kBlock >= bytes) break;
                    const int left = (int)bytes - (int)(off + i * kBlock + j * 16);
                    const auto wa = operand<DT>(now.of_a(i, left)), wb = operand<DT>(now.of_b(i, left));
                    const char *const x = cols + (half * kAhead + i) * (P::piece / (kChunk / kBlock)) + j * (P::piece / (kChunk / 16));
                    const auto col = [&](int q) {
                        const char *const at = x + (q * 8 + g) * P::row;
                        if constexpr (DT == SIFAR_BF16) return *reinterpret_cast<const uint4 *>(at);
                        else return Parts{*reinterpret_cast<const uint2 *>(at), *reinterpret_cast<const uint2 *>(at + P::piece), *reinterpret_cast<const uint2 *>(at + 2 * P::piece)};
                    };
#pragma unroll
                    for (int q = 0; q < G; q += 2) {
                        if ((uint32_t)q >= groups) break;
                        if constexpr (DT == SIFAR_F32) multiply_block<2>(acc + q, less + q, wa, wb, {col(q), col(q + 1)});
                        else multiply_block<2>(acc + q, wa, wb, {col(q), col(q + 1)});
                        if constexpr (P::parts == 2) multiply_block<2>(acc + q + G, wa, wb, {col(q + G), col(q + 1 + G)});
                    }
                }
            }
            if constexpr (DT == SIFAR_F32) {                        /* a chunk's sums */
#pragma unroll
                for (int q = 0; q < G; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sum[q][i] += acc[q][i] + less[q][i];
                        acc[q][i] = less[q][i] = 0.0f;
                    }
            }
        }
        /* rows g (first) and g + 8 (second) of the warp's 16, token t of the pass */
        auto put = [&](uint32_t t, float first, float second) {
            if (t >= n) return;
            const size_t to = at.first + t;
            if (DOWN) {
                const uint32_t r = at.tile * 128 + warp * 16 + g;
                float *const y = a.y + to * a.hidden + r;
                if (r < a.hidden) y[0] = first;
                if (r + 8 < a.hidden) y[8] = second;
            } else {
                const uint32_t r = at.tile * 64 + warp * 8 + g;
                if (r >= a.inter) return;
                const float v = weight_of(a, s_token[to], at.expert) * (activate(first, a.activation) * second);
                store_h<DT == SIFAR_BF16 ? 2 : 3>(a, a.h + to * (DT == SIFAR_BF16 ? 2 : 3) * a.h_row, a.h_row, r, v);
            }
        };
#pragma unroll
        for (int q = 0; q < G; ++q) {
            if ((uint32_t)q >= groups) break;
            if constexpr (DT == SIFAR_F32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[q][i] = sum[q][i];
            }
            if (P::parts == 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[q][i] += acc[(q + G) % P::groups][i];
            }
            put(q * 8 + 2 * j, acc[q][0], acc[q][2]);
            put(q * 8 + 2 * j + 1, acc[q][1], acc[q][3]);
        }
    }
}

/* The tokens' rows once more, on 16-byte boundaries, zeros behind their ends; binary32 ones as their three parts. */
template <int DT>
__global__ void __launch_bounds__(kThreads) k_align(const __grid_constant__ ExpertsArgs a)
{
    const uint32_t row = (a.hidden * 2 + 15u) & ~15u, at = (blockIdx.x * kThreads + threadIdx.x) * 16;      /* of bf16 values */
    grid_wait();
    grid_let_next_in();
    if (at >= row) return;
    const char *const x = a.x + blockIdx.y * a.ld_x;
    char *const to = a.rows + (size_t)blockIdx.y * (DT == SIFAR_F32 ? 3 : 1) * row + at;
    if constexpr (DT == SIFAR_BF16) {
        *reinterpret_cast<uint4 *>(to) = load_shifted(x + at, a.hidden * 2 - at);
    } else {
        uint4 v[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t c = at / 2 + 4 * i;
            const auto get = [&](uint32_t col) { return col < a.hidden ? reinterpret_cast<const uint32_t *>(x)[col] : 0u; };
            v[i] = make_uint4(get(c), get(c + 1), get(c + 2), get(c + 3));
        }
        const Parts p = parts_of(v[0]), q = parts_of(v[1]);
        *reinterpret_cast<uint4 *>(to) = make_uint4(p.high.x, p.high.y, q.high.x, q.high.y);
        *reinterpret_cast<uint4 *>(to + row) = make_uint4(p.mid.x, p.mid.y, q.mid.x, q.mid.y);
        *reinterpret_cast<uint4 *>(to + 2 * row) = make_uint4(p.low.x, p.low.y, q.low.x, q.low.y);
    }
}

/* out_t = the sum over its choices here, in their order; a second choice of the same expert has its share in the first. */
template <int DT>
__global__ void __launch_bounds__(kThreads) k_gather(const __grid_constant__ ExpertsArgs a)
{
    __shared__ int s_row[SIFAR_ROUTE_MAX_TOP_K];
    const uint32_t t = blockIdx.y, c0 = (blockIdx.x * kThreads + threadIdx.x) * 4;
    const uint32_t mine = t * a.top_k + threadIdx.x;
    int row = threadIdx.x < a.top_k && expert_of(a, mine) >= 0 ? 0 : -1;                 /* the choices were complete long ago */
    grid_wait();
    grid_let_next_in();
    if (row >= 0) row = __ldcg(a.place + mine);
    if (threadIdx.x < a.top_k) s_row[threadIdx.x] = row;
    __syncthreads();
    if (c0 >= a.hidden) return;
    float v[4] = {};
    const bool vec = a.hidden % 4 == 0;
#pragma unroll 4
    for (uint32_t k = 0; k < a.top_k; ++k) {
        if (s_row[k] < 0) continue;
        const float *const y = a.y + (size_t)s_row[k] * a.hidden + c0;
        if (vec) {
            const float4 w = __ldcg(reinterpret_cast<const float4 *>(y));
            v[0] += w.x; v[1] += w.y; v[2] += w.z; v[3] += w.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c0 + i < a.hidden) v[i] += __ldcg(y + i);
        }
    }
    auto *const out = reinterpret_cast<typename Elem<DT>::type *>(a.out + t * a.ld_out) + c0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c0 + i < a.hidden) out[i] = narrow<DT>(v[i]);
}

/* ------------------------------------------------------------------------ */
/* host                                                                      */
/* ------------------------------------------------------------------------ */
struct ExpertsPlan { bool few; uint32_t x_row, h_row; size_t h_bytes, y_bytes, rows_bytes, bytes; };

static int plan_experts(const char *fn, const sifar_experts_args *g, ExpertsPlan &p)
{
    if (!g) { set_error("%s: no argument block", fn); return SIFAR_ERR_INVALID; }
    if ((g->dtype != SIFAR_BF16 && g->dtype != SIFAR_F32) || g->experts < 1 || g->experts > SIFAR_ROUTE_MAX_EXPERTS || g->top_k < 1 ||
        g->top_k > SIFAR_ROUTE_MAX_TOP_K || (g->activation != SIFAR_ACT_SILU && g->activation != SIFAR_ACT_GELU)) {
        set_error("%s: need dtype in {0,1}, 1 <= experts <= %d, 1 <= top_k <= %d and a known activation", fn, (int)SIFAR_ROUTE_MAX_EXPERTS, (int)SIFAR_ROUTE_MAX_TOP_K);
        return SIFAR_ERR_INVALID;
    }
    if (g->tokens > SIFAR_EXPERTS_MAX_TOKENS || g->hidden < 1 || g->hidden > SIFAR_EXPERTS_MAX_COLS || g->inter < 1 || g->inter > SIFAR_EXPERTS_MAX_COLS) {
        set_error("%s: need tokens of at most %d, hidden and inter of 1 .. %d", fn, (int)SIFAR_EXPERTS_MAX_TOKENS, (int)SIFAR_EXPERTS_MAX_COLS);
        return SIFAR_ERR_INVALID;
    }
    const size_t es = elem_size(g->dtype), T = g->tokens, choices = T * (size_t)g->top_k, parts = g->dtype == SIFAR_BF16 ? 2 : 1;
    /* a multiple of 128 bytes and 64 more: two rows' pieces lie in different banks */
    p.x_row = (uint32_t)((g->hidden * es + 127) / 128 * 128 + 64);
    const bool tiles = g->dtype == SIFAR_BF16 && g->hidden % 8 == 0 && g->inter % 8 == 0;      /* as far as the sizes go */
    const size_t most = choices < (size_t)g->experts ? choices : (size_t)g->experts;       /* experts that can have tokens */
    /* Up to 16 tokens every expert may as well take them all as columns (binary32, 12 tokens, 32 experts of 512 x 1024: 56 us, 62 with each
       expert's own); up to 32 where the experts' own would leave SMs without rows (20 tokens, 8 experts of 173 x 701: 31 us, 61), but
       not where they don't (31 tokens, 64 experts of 1000 x 512: 227 us, 104; bf16, 1000 x 1022: 169 us, 141). */
    const bool all_sms = most * ((g->hidden + 127) / 128) >= kSms && most * ((g->inter + 63) / 64) >= kSms;
    const size_t limit = tiles ? kFew : all_sms ? kFewMost / 2 : kFewMost;
    p.few = T <= limit && (T + 3) / 4 * 4 * p.x_row <= (T <= (size_t)kFew ? kFewShared : kFewMostShared);
    /* binary32: a few tokens' products as they are, else three bf16 parts */
    const size_t h_parts = parts == 2 ? 2 : p.few ? 1 : 3, row2 = (g->hidden * 2 + 15) / 16 * 16;
    p.h_row = (uint32_t)((g->inter * (h_parts == 1 ? 4 : 2) + 15) / 16 * 16);
    p.h_bytes = ((p.few ? most * T : choices) * h_parts * p.h_row + 15) / 16 * 16;
    p.y_bytes = p.few ? 0 : (choices * g->hidden * sizeof(float) + 15) / 16 * 16;
    p.rows_bytes = p.few ? 0 : T * (parts == 2 ? 1 : 3) * row2;
    p.bytes = p.h_bytes + p.y_bytes + p.rows_bytes + (p.few ? 0 : choices * sizeof(int));
    return SIFAR_OK;
}

static cudaError_t launch_shared(void (*kernel)(ExpertsArgs), dim3 grid, size_t shared, cudaStream_t stream, unsigned cluster, const ExpertsArgs &a)
{
    if (shared)                              /* with what the kernels declare themselves it may be more than 48 KB */
        if (cudaError_t e = cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared)) return e;
    return launch_op(kernel, grid, dim3(kThreads), cluster, shared, stream, a);
}
static cudaError_t launch_shared(void (*kernel)(ExpertsArgs), dim3 grid, size_t shared, cudaStream_t stream, const ExpertsArgs &a)
{
    return launch_shared(kernel, grid, shared, stream, 1, a);
}

template <int DT, int G>
static cudaError_t launch_few(const ExpertsPlan &p, bool gu_vec, bool dn_vec, bool x_vec, cudaStream_t stream, ExpertsArgs a)
{
    const size_t shared = (a.tokens + 3) / 4 * 4 * (size_t)p.x_row, staged = (size_t)kWarps * 2 * Staged<DT, G>::bytes;
    const unsigned ctas = kSms * few_ctas<G>(shared);
    cudaError_t e = !gu_vec ? launch_shared(k_up_few<DT, G, false, false>, dim3(ctas), shared, stream, a)
                    : x_vec ? launch_shared(k_up_few<DT, G, true, true>, dim3(ctas), shared, stream, a) : launch_shared(k_up_few<DT, G, true, false>, dim3(ctas), shared, stream, a);
    if (e) return e;
    /* Blocks of up to 16 columns.  Where they would leave half of the CTAs without work, clusters share them, each warp two items at
       least: of 8 columns per block only half of a warp's loads are under way.  Between that and all CTAs, blocks of 8 to 16. */
    const unsigned most = kSms * kFewCtas<G>, full = (a.hidden + 15) / 16;
    const size_t pieces = ((size_t)a.inter * elem_size(DT) + kAhead * kBlock - 1) / (kAhead * kBlock), choices = (size_t)a.tokens * a.top_k;
    const size_t items = (choices < a.experts ? choices : a.experts) * pieces;
    a.split = 1;
    while (a.split < kMaxSplit && 2 * a.split * full <= most && 2 * 2 * a.split * kWarps <= items) a.split *= 2;
    const unsigned half = (a.hidden + 7) / 8, columns = a.split > 1 ? full : half < most ? half : most;
    const auto down = [&](auto kernel, size_t bytes) { return launch_shared(kernel, dim3(columns * a.split), bytes, stream, a.split, a); };
    if constexpr (DT == SIFAR_BF16 && G == 1) {
        if (a.tokens <= 4) return dn_vec ? down(k_down_few<DT, G, true, true>, 0) : down(k_down_few<DT, G, false, true>, 0);
    }
    return dn_vec ? down(k_down_few<DT, G, true, false>, staged) : down(k_down_few<DT, G, false, false>, staged);
}

template <int DT>
static cudaError_t launch_experts(const ExpertsPlan &p, bool gu_vec, bool dn_vec, bool x_vec, cudaStream_t stream, ExpertsArgs a)
{
    const dim3 grid(2 * kSms);
    cudaError_t e;
    if (p.few) {
        if (a.tokens <= 8) return launch_few<DT, 1>(p, gu_vec, dn_vec, x_vec, stream, a);
        return a.tokens <= 16 ? launch_few<DT, 2>(p, gu_vec, dn_vec, x_vec, stream, a) : launch_few<DT, 4>(p, gu_vec, dn_vec, x_vec, stream, a);
    }
    if (DT == SIFAR_F32 || !x_vec) {         /* the products below take the tokens' rows in whole pieces of bf16 values */
        const ExpertsArgs rows = a;
        const unsigned row = (a.hidden * 2 + 15) / 16 * 16;
        a.x = a.rows; a.ld_x = (DT == SIFAR_F32 ? 3 : 1) * row;
        e = launch_shared(k_align<DT>, dim3((row / 16 + kThreads - 1) / kThreads, a.tokens), 0, stream, rows);
        if (e) return e;
    }
    if (DT == SIFAR_BF16 && gu_vec && dn_vec) {
        e = launch_expert_tiles(stream, a);
        if (e) return e;
        return launch_shared(k_gather<DT>, dim3((a.hidden + 4 * kThreads - 1) / (4 * kThreads), a.tokens), 0, stream, a);
    }
    const size_t bits = (size_t)a.experts * ((a.tokens + 31) / 32) * sizeof(uint32_t);
    const auto shared = [&](size_t columns) { return columns > bits ? columns : bits; };
    e = gu_vec ? launch_shared(k_products<DT, false, true>, grid, shared(Pass<DT, false>::shared), stream, a)
               : launch_shared(k_products<DT, false, false>, grid, shared(Pass<DT, false>::shared), stream, a);
    if (e) return e;
    e = dn_vec ? launch_shared(k_products<DT, true, true>, grid, shared(Pass<DT, true>::shared), stream, a)
               : launch_shared(k_products<DT, true, false>, grid, shared(Pass<DT, true>::shared), stream, a);
    if (e) return e;
    return launch_shared(k_gather<DT>, dim3((a.hidden + 4 * kThreads - 1) / (4 * kThreads), a.tokens), 0, stream, a);
}

}  /* namespace sifar */

using namespace sifar;

extern "C" size_t sifar_experts_workspace(const sifar_experts_args *g)
{
    ExpertsPlan p;
    return plan_experts("sifar_experts_workspace", g, p) == SIFAR_OK ? p.bytes : 0;
}

extern "C" int sifar_experts(const sifar_experts_args *g, void *stream)
{
    static const char *fn = "sifar_experts";
    ExpertsPlan p;
    if (int rc = plan_experts(fn, g, p)) return rc;
    if (g->tokens == 0) return SIFAR_OK;
    if (!g->x || !g->indices || !g->weights || !g->gate_up || !g->down || !g->out) {
        set_error("%s: x, indices, weights, gate_up, down and out are needed", fn);
        return SIFAR_ERR_INVALID;
    }
    if (!g->workspace || (uintptr_t)g->workspace % 16 || g->workspace_bytes < p.bytes) {
        set_error("%s: needs %zu bytes of workspace on a 16-byte boundary", fn, p.bytes);
        return SIFAR_ERR_INVALID;
    }
    const size_t es = elem_size(g->dtype), T = g->tokens, H = g->hidden, I = g->inter, E = (size_t)g->experts, choices = T * (size_t)g->top_k;
    const auto ld = [](size_t given, size_t cols) { return given ? given : cols; };
    const RowArray all[] = {
        RowArray{"x", g->x, T, H, ld(g->ld_x, H), es, false},
        RowArray{"indices", g->indices, 1, choices, choices, sizeof(int), false},
        RowArray{"weights", g->weights, 1, choices, choices, sizeof(float), false},
        RowArray{"gate_up", g->gate_up, E * 2 * I, H, ld(g->ld_gate_up, H), es, false},
        RowArray{"down", g->down, E * H, I, ld(g->ld_down, I), es, false},
        RowArray{"out", g->out, T, H, ld(g->ld_out, H), es, true},
        RowArray{"workspace", g->workspace, 1, p.bytes, p.bytes, 1, true},
    };
    if (int rc = check_arrays(fn, all, 7)) return rc;
    ExpertsArgs a;
    a.x = (const char *)g->x; a.gate_up = (const char *)g->gate_up; a.down = (const char *)g->down; a.out = (char *)g->out;
    a.indices = g->indices; a.weights = g->weights;
    a.h = (char *)g->workspace; a.y = (float *)((char *)g->workspace + p.h_bytes); a.rows = (char *)a.y + p.y_bytes; a.place = (int *)(a.rows + p.rows_bytes);
    a.ld_x = all[0].ld * es; a.ld_gate_up = all[3].ld * es; a.ld_down = all[4].ld * es; a.ld_out = all[5].ld * es;
    a.tokens = (uint32_t)T; a.hidden = (uint32_t)H; a.inter = (uint32_t)I; a.h_row = p.h_row; a.top_k = (uint32_t)g->top_k;
    a.experts = (uint32_t)E; a.first = g->first_expert; a.activation = g->activation; a.x_row = p.x_row;
    const bool gu = rows_aligned16(all[3]) && H * es % 16 == 0, dn = rows_aligned16(all[4]) && I * es % 16 == 0, xv = rows_aligned16(all[0]) && H * es % 16 == 0;
    const cudaError_t err = g->dtype == SIFAR_BF16 ? launch_experts<SIFAR_BF16>(p, gu, dn, xv, (cudaStream_t)stream, a)
                                                   : launch_experts<SIFAR_F32>(p, gu, dn, xv, (cudaStream_t)stream, a);
    SIFAR_CUDA(err);
    return SIFAR_OK;
}
