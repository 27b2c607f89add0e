/*
 * sifar_attention.cu - attention of one new token per sequence over a paged cache, split over the cache's length.
 *
 * An item is a key head of a sequence with up to 16 (binary32: 8) of the query heads that read it.  All items' strips of 16
 * tokens in a row are cut into equal shares, one per team, whatever the lengths: a team goes through the end of one item, some
 * whole ones and the start of another without meeting any other team.  Its strips come through a ring of its own in shared
 * memory, filled by asynchronous 16-byte copies two strips ahead, across items too; an item's queries come the same way, before
 * its strips.  An item that several teams had is put together by a second kernel from their maxima, sums and weighted values;
 * where a CTA's teams all have the same item they join their parts first.
 *
 * A team is a warp, and where an item has more than eight query heads in bf16 two warps, eight heads each, that fill and read the
 * same ring (48 users with a window of 1000 and 16 heads of 256: 24.5 us, with all 16 in one warp 31).
 *
 * Scores and weighted values are matrix instructions in bf16, the tokens' rows as they lie in the ring; a strip's exponentials
 * go into the second product as two bf16 values, the rounded one and what it leaves (16 bits).  binary32 has its
 * sums from fused multiply-adds.  Maxima, sums and values are binary32 from the first strip to the join.
 *
 * Bound by the memory where there is enough of it: two users with 131072 tokens of 8 x 128 171 us, 6.3 TB/s; 64 users of up to
 * 8192 tokens 46 us, 5.0 TB/s, of which about 10 are the start, the uneven ends and the second kernel; one user with 2000 tokens
 * 11.0 us, no more than those.  binary32 is bound by latencies (37 users of up to 1777 tokens, heads of 80: 19.4 us, 1.4 TB/s): the rings leave an
 * SM one CTA of four warps, whose schedulers issue in 26 % of the cycles.
 */
#include "sifar_cache.cuh"
#include "sifar_norm_shape.cuh"

namespace sifar {

constexpr int kTeams = 4;                    /* of a CTA */
constexpr int kItemCost = 1;                 /* what an item's start and end count as, in strips */
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

/* Where a split item lies in the workspace: partials of teams first .. last, in the order of the tokens. */
struct Split { int sequence, item, first, last, slot, one0, one1, pad; };
/* slot: of `first`'s partial, 0 of the others; first < 0: none.  Teams one0 .. one1 - 1 are whole CTAs that left one partial each, in
   the place of their first team. */

struct AttentionArgs {
    const char *q, *k, *v;
    char *out;
    float *lse;
    const int *lengths;
    Pages pages;
    Split *splits;                           /* one per team */
    float *partial;                          /* team x 2 partials */
    unsigned long long ld_q, ld_out;         /* bytes */
    uint32_t sequences, window, limit;       /* limit = max_pages * page_size */
    uint32_t heads, kv_heads, group, chunks, rows, dim;   /* rows = query heads of an item, chunks of them per key head */
    float scale;                             /* times log2(e) */
    bool q_vec, out_vec;                     /* rows of q in 16-byte pieces; rows of out in pieces of four elements */
};

/* Floats of a partial: rows x dim_pad values, rows maxima, rows sums; the next one starts on 16 bytes again. */
__host__ __device__ __forceinline__ size_t partial_floats(uint32_t rows, int dim_pad) { return ((size_t)rows * (dim_pad + 2) + 3) / 4 * 4; }

/* First visible token and the one behind the last.  The window ends at the sequence's length, also where the table does not reach it. */
__device__ __forceinline__ void visible(const AttentionArgs &a, uint32_t s, uint32_t &lo, uint32_t &hi)
{
    const uint32_t n = (uint32_t)max(a.lengths[s], 0);
    hi = min(n, a.limit);
    lo = a.window && n > a.window ? min(n - a.window, hi) : 0u;
}
template <int TOKENS> __device__ __forceinline__ uint32_t strips_of(uint32_t lo, uint32_t hi)
{
    return max(1u, (hi - lo + TOKENS - 1) / TOKENS);     /* an empty sequence has an item too: its zeros */
}

/* A quotient that mostly fits 32 bits. */
__device__ __forceinline__ unsigned long long quotient(unsigned long long n, uint32_t d)
{
    return n >> 32 ? n / d : (unsigned long long)((uint32_t)n / d);
}

/* Where in the row of all items' strips (each followed by kItemCost places without one) a team is. */
template <int TOKENS> struct Cursor {
    unsigned long long at;                   /* place in the row */
    uint32_t sequence, item, strip;          /* item: key head and chunk of its query heads */
    uint32_t lo, hi, strips;                 /* of the sequence */

    __device__ __forceinline__ void enter(const AttentionArgs &a)
    {
        lo = hi = 0;
        if (sequence < a.sequences) visible(a, sequence, lo, hi);
        strips = strips_of<TOKENS>(lo, hi);
    }
    /* Whether the next place is another item's. */
    __device__ __forceinline__ bool advance(const AttentionArgs &a, uint32_t items)
    {
        ++at;
        if (++strip < strips) return false;
        at += kItemCost;
        strip = 0;
        if (++item < items) return true;
        item = 0;
        ++sequence;
        enter(a);
        return true;
    }
};

/* The row and what of it is a team's. */
struct Shares { unsigned long long total, share; };

/*
 * Every thread adds up the places of a run of sequences; the one whose run holds the begin of a team's share walks it.
 */
template <int TOKENS, int WARPS>
__device__ __forceinline__ Shares find_shares(const AttentionArgs &a, unsigned long long *s_sum, Cursor<TOKENS> *s_start)
{
    constexpr uint32_t threads = 32 * WARPS;
    const uint32_t run = (a.sequences + threads - 1) / threads, s0 = min(a.sequences, threadIdx.x * run), s1 = min(a.sequences, s0 + run);
    const uint32_t items = a.kv_heads * a.chunks;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    auto places = [&](uint32_t s) {
        uint32_t lo, hi;
        visible(a, s, lo, hi);
        return (unsigned long long)(strips_of<TOKENS>(lo, hi) + kItemCost) * items;
    };
    unsigned long long mine = 0;
    for (uint32_t s = s0; s < s1; ++s) mine += places(s);
    unsigned long long sum = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(0xFFFFFFFFu, sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 31) s_sum[warp] = sum;
    __syncthreads();
    unsigned long long before = 0;
    Shares r{0, 0};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) before += s_sum[w];
        r.total += s_sum[w];
    }
    before += sum - mine;
    r.share = quotient(r.total + gridDim.x * kTeams - 1, gridDim.x * kTeams);
#pragma unroll
    for (int w = 0; w < kTeams; ++w) {
        const unsigned long long begin = r.share * (blockIdx.x * kTeams + w);
        if (begin < before || begin >= before + mine) continue;
        Cursor<TOKENS> c;
        unsigned long long here = before;
        for (c.sequence = s0; c.sequence + 1 < s1; ++c.sequence) {
            const unsigned long long n = places(c.sequence);
            if (begin < here + n) break;
            here += n;
        }
        c.enter(a);
        c.item = (uint32_t)quotient(begin - here, c.strips + kItemCost);
        c.strip = (uint32_t)(begin - here - (unsigned long long)c.item * (c.strips + kItemCost));
        c.at = begin;
        if (c.strip >= c.strips) {           /* between two items: on to the next */
            c.at += c.strips + kItemCost - c.strip - 1;
            c.strip = c.strips;
            c.at -= kItemCost;
            c.advance(a, items);
        }
        s_start[w] = c;
    }
    __syncthreads();
    return r;
}

__device__ __forceinline__ uint32_t shared_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
/* `bytes` (16 or 0) from global memory, the rest of the 16 zeros. */
__device__ __forceinline__ void copy16(uint32_t to, const void *from, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_turned(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void multiply(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
/* Two values as bf16, the first in the low half, and what that leaves of them, as bf16 again. */
__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t rest_bf16(float lo, float hi, uint32_t taken)
{
    return pair_bf16(lo - __uint_as_float(taken << 16), hi - __uint_as_float(taken & 0xFFFF0000u));
}

/* A strip of keys and one of values in a warp's ring. */
template <int DT, int DP> struct Ring {
    static constexpr int es = DT == SIFAR_BF16 ? 2 : 4;
    static constexpr int tokens = DP * es > 512 ? 8 : 16;           /* of a strip */
    static constexpr int row = DP * es, chunks = row / 16;          /* bytes, 16-byte pieces of a row */
    static constexpr int strip = tokens * row;                      /* keys or values */
    static constexpr int stages = DP * es <= 128 ? 4 : 3;
    static constexpr int bytes = stages * 2 * strip;
    /* Pieces of a row change places by its number so that what is read at once lies in different banks: binary32 lanes read two
       (tokens = 8: four) pieces of each row, ldmatrix one piece of eight rows. */
    static __device__ __forceinline__ int place(int r, int piece)
    {
        return piece ^ (DT == SIFAR_BF16 ? r & 7 : (r * (32 / tokens)) & 7);
    }
};

/* Issues the copies of a strip, a warp of a team its part of the tokens.  `offset` is that of token lane % tokens, -1 if it is masked. */
template <int DT, int DP, int TW, bool VEC>
__device__ __forceinline__ void fetch(const AttentionArgs &a, char *ring, int stage, long long offset, unsigned long long head, int sub)
{
    using R = Ring<DT, DP>;
    const int lane = threadIdx.x & 31;
    char *const ks = ring + stage * 2 * R::strip, *const vs = ks + R::strip;
    if (VEC) {
        /* R::chunks lanes per row */
        constexpr int rows = 32 / R::chunks > 0 ? 32 / R::chunks : 1, per = R::chunks > 32 ? R::chunks / 32 : 1;
#pragma unroll
        for (int i = 0; i < R::tokens / TW; i += rows) {
            const int r = sub * (R::tokens / TW) + i + (R::chunks >= 32 ? 0 : lane / R::chunks);
            const long long at = __shfl_sync(0xFFFFFFFFu, offset, r);
#pragma unroll
            for (int c = 0; c < per; ++c) {
                const int piece = (R::chunks >= 32 ? lane : lane % R::chunks) + 32 * c;
                const bool there = at >= 0 && (uint32_t)(piece * 16) < a.dim * R::es;
                const unsigned long long from = there ? (unsigned long long)at + head + piece * 16 : 0ull;
                const int to = r * R::row + R::place(r, piece) * 16;
                copy16(shared_at(ks + to), a.k + from, there ? 16u : 0u);
                copy16(shared_at(vs + to), a.v + from, there ? 16u : 0u);
            }
        }
    } else {
        using T = typename Elem<DT>::type;
#pragma unroll 1
        for (int r = sub * (R::tokens / TW); r < (sub + 1) * (R::tokens / TW); ++r) {
            const long long at = __shfl_sync(0xFFFFFFFFu, offset, r);
            T k[DP / 32], v[DP / 32];
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) {
                const uint32_t d = i * 32 + lane;
                const bool there = at >= 0 && d < a.dim;
                const unsigned long long from = there ? (unsigned long long)at + head + d * R::es : 0ull;
                k[i] = there ? *reinterpret_cast<const T *>(a.k + from) : (T)0;
                v[i] = there ? *reinterpret_cast<const T *>(a.v + from) : (T)0;
            }
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) {
                const int d = (i * 32 + lane) * R::es, to = r * R::row + R::place(r, d / 16) * 16 + d % 16;
                *reinterpret_cast<T *>(ks + to) = k[i];
                *reinterpret_cast<T *>(vs + to) = v[i];
            }
        }
    }
}

/* Issues the copies of an item's queries r0 .. r0 + ROWS - 1, into the place of a strip's keys: row r of them where token r's key would lie. */
template <int DT, int DP, int ROWS>
__device__ __forceinline__ void fetch_queries(const AttentionArgs &a, char *ring, int stage, const char *q, uint32_t rows, uint32_t r0)
{
    using R = Ring<DT, DP>;
    char *const to = ring + stage * 2 * R::strip;
    const uint32_t lane = threadIdx.x & 31, row = a.dim * R::es;
    if (a.q_vec) {
#pragma unroll 4
        for (uint32_t i = lane; i < ROWS * R::chunks; i += 32) {
            const uint32_t r = r0 + i / R::chunks, piece = i % R::chunks;
            const bool there = r < rows && piece * 16 < row;
            copy16(shared_at(to + r * R::row + R::place(r, piece) * 16), a.q + (there ? q - a.q + (r * row + piece * 16) : 0), there ? 16u : 0u);
        }
    } else {
        using T = typename Elem<DT>::type;
#pragma unroll 4
        for (uint32_t i = lane; i < ROWS * DP; i += 32) {
            const uint32_t r = r0 + i / DP, d = i % DP;
            *reinterpret_cast<T *>(to + r * R::row + R::place(r, d * R::es / 16) * 16 + d * R::es % 16) =
                r < rows && d < a.dim ? reinterpret_cast<const T *>(q)[r * a.dim + d] : (T)0;
        }
    }
}

/* A maximum of -infinity says that there is nothing; NaN scores alone leave that too, but a sum of NaN. */
__device__ __forceinline__ float top_of(float top, float sum) { return sum != sum ? NAN : top; }

/* Where four values of a row lie when a state is left in shared memory: rows are shifted against one another by pieces. */
template <int DP> __device__ __forceinline__ int value_place(int row, int piece) { return row * DP + ((piece ^ (row & 7)) * 4); }

/* ------------------------------------------------------------------------ */
/* what a warp holds of an item                                              */
/* ------------------------------------------------------------------------ */
/*
 * bf16: matrix instructions of 16 rows x 16 x 8.  A warp's eight query heads take the upper half of the rows, and the
 * probabilities go in as two bf16 values, the rounded one above and what it leaves below: they keep 16 bits at no further
 * instruction.
 */
template <int DP> struct StateBf16 {
    using R = Ring<SIFAR_BF16, DP>;
    uint32_t q[DP / 16][2];
    float o[DP / 8][4];
    float m, l;                                     /* l: this lane's columns */

    __device__ __forceinline__ void clear()
    {
        m = -INFINITY; l = 0.0f;
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    }
    /* From the queries' place in the ring, rows r0 .. r0 + 7. */
    __device__ __forceinline__ void begin(const char *ring, int stage, int r0, float *)
    {
        const int lane = threadIdx.x & 31, row = r0 + (lane & 7);
        const uint32_t qs = shared_at(ring + stage * 2 * R::strip);
        clear();
#pragma unroll
        for (int i = 0; i < DP / 16; i += 2) {      /* four pieces at a time */
            uint32_t b[4];
            load_matrices(b, qs + row * R::row + R::place(row, 2 * i + (lane >> 3)) * 16);
            q[i][0] = b[0]; q[i][1] = b[1]; q[i + 1][0] = b[2]; q[i + 1][1] = b[3];
        }
    }

    /* seen: bit t set where token t of the strip counts */
    __device__ __forceinline__ void strip(const AttentionArgs &a, const char *ring, int stage, uint32_t seen, float *)
    {
        const int lane = threadIdx.x & 31, j = lane & 3;
        const uint32_t ks = shared_at(ring + stage * 2 * R::strip), vs = ks + R::strip;
        float s[2][4] = {}, s2[2][4] = {};                          /* two chains of sums each */
        {
            const int row = (lane & 7) + ((lane >> 4) & 1) * 8, half = (lane >> 3) & 1;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                uint32_t b[4];
                load_matrices(b, ks + row * R::row + R::place(row, 2 * i + half) * 16);
                float (&c)[2][4] = i & 1 ? s2 : s;
                multiply(c[0], q[i][0], 0u, q[i][1], 0u, b[0], b[1]);
                multiply(c[1], q[i][0], 0u, q[i][1], 0u, b[2], b[3]);
            }
        }
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = seen >> ((i >> 1) * 8 + 2 * j + (i & 1)) & 1u;
            x[i] = in ? (s[i >> 1][i & 1] + s2[i >> 1][i & 1]) * a.scale : -INFINITY;
        }
        float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const float now = fmaxf(m, top), ref = now == -INFINITY ? 0.0f : now, keep = exp2f(m - ref);
        m = now;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = exp2f(x[i] - ref);
        l = l * keep + ((x[0] + x[1]) + (x[2] + x[3]));
        uint32_t p[2], rest[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            p[i] = pair_bf16(x[2 * i], x[2 * i + 1]);
            rest[i] = rest_bf16(x[2 * i], x[2 * i + 1], p[i]);
        }
        if (__any_sync(0xFFFFFFFFu, keep != 1.0f)) {
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) { o[i][0] *= keep; o[i][1] *= keep; o[i][2] *= keep; o[i][3] *= keep; }
        }
        const int row = lane & 15, half = lane >> 4;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            uint32_t b[4];
            load_matrices_turned(b, vs + row * R::row + R::place(row, 2 * i + half) * 16);
            multiply(o[2 * i], p[0], rest[0], p[1], rest[1], b[0], b[1]);
            multiply(o[2 * i + 1], p[0], rest[0], p[1], rest[1], b[2], b[3]);
        }
    }

    /* Values (rows x DP, pieces of four in changed places), maxima and sums of rows r0 .. r0 + 7 into shared memory. */
    __device__ __forceinline__ void leave(float *values, int r0, float *tops, float *sums)
    {
        const int lane = threadIdx.x & 31, j = lane & 3, row = r0 + (lane >> 2);
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
        if (j == 0) { tops[row] = top_of(m, l); sums[row] = l; }
#pragma unroll
        for (int i = 0; i < DP / 8; ++i)
            *reinterpret_cast<float2 *>(values + value_place<DP>(row, 2 * i + (j >> 1)) + (j & 1) * 2) = make_float2(o[i][0] + o[i][2], o[i][1] + o[i][3]);
    }
};

/*
 * binary32: products by ordinary instructions.  For the scores two lanes (DP = 256: four) share a token and take every other
 * 16-byte piece of its key; the queries come from shared memory.  For the values a lane holds 4 (8) columns of all heads and walks
 * the strip's tokens.
 */
template <int DP, int ROWS> struct StateF32 {
    using R = Ring<SIFAR_F32, DP>;
    static constexpr int L = 32 / R::tokens;                        /* lanes of a token */
    static constexpr int half = DP < 128 ? 2 : 1;                   /* halves of the warp with tokens of their own (values) */
    static constexpr int C = DP / (128 / half);                     /* pieces of a lane */
    float o[ROWS][C][4];
    float m[ROWS], l[ROWS];
    const float *q;

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int h = 0; h < ROWS; ++h) {
            m[h] = -INFINITY; l[h] = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c) o[h][c][0] = o[h][c][1] = o[h][c][2] = o[h][c][3] = 0.0f;
        }
    }
    __device__ __forceinline__ void begin(const char *ring, int stage, int, float *q_shared)
    {
        clear();
        q = q_shared;
        const char *const qs = ring + stage * 2 * R::strip;
#pragma unroll 4
        for (int i = threadIdx.x & 31; i < ROWS * R::chunks; i += 32) {
            const int r = i / R::chunks, piece = i % R::chunks;
            *reinterpret_cast<float4 *>(q_shared + r * DP + piece * 4) = *reinterpret_cast<const float4 *>(qs + r * R::row + R::place(r, piece) * 16);
        }
        __syncwarp();
    }

    __device__ __forceinline__ void strip(const AttentionArgs &a, const char *ring, int stage, uint32_t seen, float *p_shared)
    {
        const int lane = threadIdx.x & 31, t = lane / L, part = lane % L;
        const char *const ks = ring + stage * 2 * R::strip, *const vs = ks + R::strip;
        float s[ROWS] = {};
        const int pieces = (int)(a.dim + 3) / 4;
#pragma unroll 4
        for (int i = part; i < pieces; i += L) {
            const float4 k = *reinterpret_cast<const float4 *>(ks + t * R::row + R::place(t, i) * 16);
#pragma unroll
            for (int h = 0; h < ROWS; ++h) {
                const float4 x = *reinterpret_cast<const float4 *>(q + h * DP + i * 4);
                s[h] += x.x * k.x; s[h] += x.y * k.y; s[h] += x.z * k.z; s[h] += x.w * k.w;
            }
        }
        const bool in = seen >> t & 1u;
        bool moved = false;
        float keep[ROWS];
#pragma unroll
        for (int h = 0; h < ROWS; ++h) {
#pragma unroll
            for (int d = 1; d < L; d <<= 1) s[h] += __shfl_xor_sync(0xFFFFFFFFu, s[h], d);
            s[h] = in ? s[h] * a.scale : -INFINITY;
            float top = s[h];
#pragma unroll
            for (int d = L; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            const float now = fmaxf(m[h], top), ref = now == -INFINITY ? 0.0f : now;
            keep[h] = exp2f(m[h] - ref);
            moved = moved || keep[h] != 1.0f;
            m[h] = now;
            const float p = exp2f(s[h] - ref);
            l[h] = l[h] * keep[h] + (part == 0 ? p : 0.0f);
            if (part == 0) p_shared[h * R::tokens + t] = p;
        }
        __syncwarp();
        if (moved) {                                                /* all lanes have the same */
#pragma unroll
            for (int h = 0; h < ROWS; ++h)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[h][c][e] *= keep[h];
        }
        const int piece = half == 2 ? lane & 15 : lane, first = half == 2 ? (lane >> 4) * 4 : 0;
#pragma unroll 1
        for (int t0 = first; t0 < R::tokens; t0 += 4 * half) {
            float4 v[4][C];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int c = 0; c < C; ++c) v[e][c] = *reinterpret_cast<const float4 *>(vs + (t0 + e) * R::row + R::place(t0 + e, piece + 32 * c) * 16);
#pragma unroll
            for (int h = 0; h < ROWS; ++h) {
                const float4 p = *reinterpret_cast<const float4 *>(p_shared + h * R::tokens + t0);
                const float w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        o[h][c][0] += w[e] * v[e][c].x; o[h][c][1] += w[e] * v[e][c].y;
                        o[h][c][2] += w[e] * v[e][c].z; o[h][c][3] += w[e] * v[e][c].w;
                    }
            }
        }
        __syncwarp();
    }

    __device__ __forceinline__ void leave(float *values, int, float *tops, float *sums)
    {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int h = 0; h < ROWS; ++h) {
            const float sum = warp_sum(l[h]);
            if (lane == 0) { tops[h] = top_of(m[h], sum); sums[h] = sum; }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = half == 2 ? o[h][c][e] + __shfl_xor_sync(0xFFFFFFFFu, o[h][c][e], 16) : o[h][c][e];
                if (half == 1 || lane < 16)
                    *reinterpret_cast<float4 *>(values + value_place<DP>(h, half == 2 ? lane & 15 : lane + 32 * c)) = make_float4(x[0], x[1], x[2], x[3]);
            }
        }
    }
};

template <int DT, int DP, int ROWS> struct StateOf { using type = StateBf16<DP>; };
template <int DP, int ROWS> struct StateOf<SIFAR_F32, DP, ROWS> { using type = StateF32<DP, ROWS>; };

/* Shared memory: the rings (a team leaves its values in its own), behind them each team's binary32 queries and probabilities. */
template <int DT, int DP, int ROWS> struct Shared {
    static constexpr int rings = kTeams * Ring<DT, DP>::bytes;
    static constexpr int per_team = DT == SIFAR_F32 ? ROWS * (DP + Ring<DT, DP>::tokens) * 4 : 0;
    static constexpr int bytes = rings + kTeams * per_team;
    static_assert(ROWS * DP * 4 <= 2 * Ring<DT, DP>::strip, "a state fits a stage");
};

/* Four values of an output row from column d on. */
template <int DT> __device__ __forceinline__ void store_out(typename Elem<DT>::type *to, const float (&x)[4], uint32_t d, uint32_t dim, bool vec)
{
    if (vec) {
        if (d >= dim) return;
        if constexpr (DT == SIFAR_BF16) *reinterpret_cast<uint2 *>(to + d) = make_uint2(pair_bf16(x[0], x[1]), pair_bf16(x[2], x[3]));
        else *reinterpret_cast<float4 *>(to + d) = make_float4(x[0], x[1], x[2], x[3]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (d + e < dim) to[d + e] = narrow<DT>(x[e]);
}

/* Warps of a team, and CTAs that an SM holds by shared memory (227 KB, 1 KB of it per CTA for the system) and by 255 registers of
   128 threads, 128 of 256. */
template <int DT, int ROWS> __host__ __device__ constexpr int team_warps() { return DT == SIFAR_BF16 && ROWS > 8 ? 2 : 1; }
template <int DT, int DP, int ROWS> __host__ __device__ constexpr int ctas_per_sm()
{
    return 227 * 1024 / (Shared<DT, DP, ROWS>::bytes + 2048) < 2 ? 1 : 2;
}

template <int DT, int DP, int ROWS, bool VEC>
__global__ void __launch_bounds__(32 * kTeams * team_warps<DT, ROWS>(), ctas_per_sm<DT, DP, ROWS>()) k_attend(const __grid_constant__ AttentionArgs a)
{
    using R = Ring<DT, DP>;
    using Sh = Shared<DT, DP, ROWS>;
    using C = Cursor<R::tokens>;
    using T = typename Elem<DT>::type;
    extern __shared__ __align__(128) char smem[];
    __shared__ unsigned long long s_sum[kTeams * team_warps<DT, ROWS>()];
    __shared__ C s_start[kTeams];
    __shared__ float s_top[kTeams][ROWS], s_l[kTeams][ROWS], s_w[kTeams][ROWS];
    constexpr int es = sizeof(T), TW = team_warps<DT, ROWS>(), own = ROWS / TW;             /* own: rows of a warp */
    const int lane = threadIdx.x & 31, team = threadIdx.x / 32 / TW, sub = TW == 1 ? 0 : threadIdx.x / 32 % TW;
    const uint32_t number = blockIdx.x * kTeams + team, items = a.kv_heads * a.chunks;
    char *const ring = smem + team * R::bytes;
    float *const q_shared = reinterpret_cast<float *>(smem + Sh::rings + team * Sh::per_team), *const p_shared = q_shared + ROWS * DP;
    const size_t part_floats = partial_floats(a.rows, DP);
    grid_let_next_in();
    grid_wait();

    /* the warps of a team meet where one warp alone would only meet its lanes */
    auto meet = [&] {
        if constexpr (TW == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" :: "r"(1 + team), "n"(32 * TW) : "memory");
    };
    if (lane == 0 && sub == 0) a.splits[number].first = -1;
    const Shares row = find_shares<R::tokens, kTeams * TW>(a, s_sum, s_start);
    const unsigned long long begin = min(row.total, row.share * number), end = min(row.total, begin + row.share);
    const bool any = begin < end;
    C now = s_start[team];                                        /* the strip to be used next */
    if (!any) now.at = end;
    /* whether all of the CTA's places belong to one item, from a strip of it on */
    const unsigned long long cta_begin = row.share * blockIdx.x * kTeams, cta_end = min(row.total, cta_begin + row.share * kTeams);
    const bool together = cta_begin < cta_end && s_start[0].at == cta_begin && cta_begin - s_start[0].strip + s_start[0].strips + kItemCost >= cta_end;

    C then = now;                                                 /* the strip to be fetched next */
    bool queries = true;                                          /* ... or the queries of its item */
    /* the lane's token of strip `then`: its page, asked for a strip ahead, and its place there */
    int page;
    uint32_t in;
    auto look_up = [&] {
        const uint32_t t = then.lo + then.strip * R::tokens + lane % R::tokens, at = page_of(a.pages, t, in);
        page = -1;
        if (then.at < end && t < then.hi && at < a.pages.max_pages) page = a.pages.table[then.sequence * a.pages.ld_table + at];
    };
    unsigned long long seen = 0;                                  /* 16 bits per stage: its tokens that count */
    look_up();
    auto fetch_next = [&](int stage) {
        if (then.at < end) {
            const uint32_t kv_head = then.item / a.chunks, chunk = then.item - kv_head * a.chunks;
            if (queries) {
                const uint32_t head = kv_head * a.group + chunk * a.rows;
                fetch_queries<DT, DP, own>(a, ring, stage, a.q + then.sequence * a.ld_q + (size_t)head * a.dim * es, min(a.rows, a.group - chunk * a.rows), sub * own);
                queries = false;
            } else {
                const long long at = place_offset(a.pages, page, in);
                queries = then.advance(a, items);
                look_up();
                seen = (seen & ~(0xFFFFull << (16 * stage))) | (unsigned long long)(__ballot_sync(0xFFFFFFFFu, at >= 0) & ((1u << R::tokens) - 1u)) << (16 * stage);
                fetch<DT, DP, TW, VEC>(a, ring, stage, at, kv_head * a.pages.stride_head, sub);
            }
        }
        copies_commit();
    };
    /* stages - 1 strips are under way before the first is used */
    for (int i = 0; i < R::stages - 1; ++i) fetch_next(i);

    typename StateOf<DT, DP, ROWS>::type state;
    state.clear();
    bool left = false, fresh = true, whole = false;                             /* whole: from the item's first strip on */
    int stage = 0;
    while (now.at < end) {
        copies_wait<R::stages - 2>();
        meet();
        fetch_next(stage == 0 ? R::stages - 1 : stage - 1);
        const int here = stage;
        stage = stage + 1 == R::stages ? 0 : stage + 1;
        if (fresh) {
            state.begin(ring, here, sub * own, q_shared);
            whole = now.strip == 0;
            fresh = false;
            continue;
        }
        state.strip(a, ring, here, (uint32_t)(seen >> (16 * here)) & 0xFFFFu, p_shared);
        const C done = now;
        now.advance(a, items);
        if (done.strip + 1 < done.strips && now.at < end) continue;

        /* the item, or this team's share of it, is done: it goes through the stage that was used last, in whole rows */
        fresh = true;
        const int values = team * R::bytes + (together ? 0 : here * 2 * R::strip);       /* in smem */
        if (together) copies_wait<0>();
        meet();
        state.leave(reinterpret_cast<float *>(smem + values), sub * own, s_top[team], s_l[team]);
        left = true;
        meet();
        const unsigned long long item_begin = done.at - done.strip;
        const bool all = whole && done.strip + 1 == done.strips;
        /* slot 0: the item that the share begins in; slot 1: one that it leaves unfinished */
        const int slot = item_begin <= begin ? 0 : 1;
        if (whole && !all && lane == 0 && sub == 0) {
            const uint32_t last = (uint32_t)quotient(item_begin + done.strips - 1, (uint32_t)row.share);
            /* CTAs from its first full one to its last that end within it, or behind it before anything else begins */
            const unsigned long long item_end = min(row.total, item_begin + done.strips + kItemCost), cta = row.share * kTeams;
            const uint32_t one0 = (uint32_t)((item_begin + cta - 1) / cta) * kTeams;
            uint32_t one1 = item_end == row.total ? (last / kTeams + 1) * kTeams : (uint32_t)(item_end / cta) * kTeams;
            one1 = max(one0, min(one1, (last / kTeams + 1) * kTeams));
            a.splits[number] = Split{(int)done.sequence, (int)done.item, (int)number, (int)last, slot, (int)one0, (int)one1, 0};
        }
        if (together && !all) break;
        const uint32_t kv_head = done.item / a.chunks, chunk = done.item - kv_head * a.chunks, rows = min(a.rows, a.group - chunk * a.rows);
        const uint32_t head = kv_head * a.group + chunk * a.rows;
        T *const out = reinterpret_cast<T *>(a.out + done.sequence * a.ld_out) + (size_t)head * a.dim;
        float *const part = a.partial + ((size_t)number * 2 + slot) * part_floats;
        const uint32_t mine = min(rows, (uint32_t)(sub + 1) * own);   /* behind the warp's last row */
        if (lane < own && sub * own + lane < (int)rows) {
            const int r = sub * own + lane;
            const float top = s_top[team][r], sum = s_l[team][r];
            s_w[team][r] = sum == 0.0f ? 0.0f : 1.0f / sum;
            if (!all) { part[a.rows * DP + r] = top; part[a.rows * DP + a.rows + r] = sum; }
            else if (a.lse) a.lse[done.sequence * (size_t)a.heads + head + r] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
        }
        meet();
        /* several loads before the first store: a warp has nobody to hide them behind */
        constexpr uint32_t kPieces = DP / 4, kAtOnce = kPieces < 32 ? 32 / kPieces : 1, kTurns = kPieces > 32 ? kPieces / 32 : 1, kRows = 4 / kTurns;
        for (uint32_t r0 = sub * own + lane / kPieces; r0 < mine; r0 += kAtOnce * kRows) {
            float4 v[kRows][kTurns];
            float f[kRows];
#pragma unroll
            for (uint32_t k = 0; k < kRows; ++k) {
                const uint32_t r = min(r0 + k * kAtOnce, mine - 1);
                f[k] = s_w[team][r];
#pragma unroll
                for (uint32_t c = 0; c < kTurns; ++c) v[k][c] = *reinterpret_cast<const float4 *>(smem + values + value_place<DP>(r, lane % kPieces + 32 * c) * 4);
            }
#pragma unroll
            for (uint32_t k = 0; k < kRows; ++k) {
                const uint32_t r = r0 + k * kAtOnce;
                if (r >= mine) break;
#pragma unroll
                for (uint32_t c = 0; c < kTurns; ++c) {
                    const uint32_t d = (lane % kPieces + 32 * c) * 4;
                    if (all) {
                        float x[4] = {v[k][c].x * f[k], v[k][c].y * f[k], v[k][c].z * f[k], v[k][c].w * f[k]};
                        if (f[k] == 0.0f) x[0] = x[1] = x[2] = x[3] = 0.0f;     /* nothing, whatever zero times the values left */
                        store_out<DT>(out + r * a.dim, x, d, a.dim, a.out_vec);
                    } else {
                        *reinterpret_cast<float4 *>(part + r * DP + d) = v[k][c];
                    }
                }
            }
        }
        meet();
    }
    copies_wait<0>();
    if (!together) return;

    /* all of the CTA's warps have strips of one item, or none: one part of them, in the first one's place */
    if (!left && lane < own) { s_top[team][sub * own + lane] = -INFINITY; s_l[team][sub * own + lane] = 0.0f; }
    __syncthreads();
    const uint32_t chunk = s_start[0].item % a.chunks, rows = min(a.rows, a.group - chunk * a.rows);
    float *const part = a.partial + (size_t)blockIdx.x * kTeams * 2 * part_floats;
    if (threadIdx.x < rows) {
        const int r = threadIdx.x;
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kTeams; ++w) top = fmaxf(top, s_top[w][r]);
        const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int w = 0; w < kTeams; ++w) {
            const float f = exp2f(s_top[w][r] - ref);
            s_w[w][r] = f;
            sum += f * s_l[w][r];
        }
        part[a.rows * DP + r] = top_of(top, sum);
        part[a.rows * DP + a.rows + r] = sum;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < rows * (DP / 4); i += 32 * kTeams * TW) {
        const uint32_t r = i / (DP / 4), piece = i % (DP / 4);
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kTeams; ++w) {
            const float f = s_w[w][r];
            const float4 o = *reinterpret_cast<const float4 *>(smem + w * R::bytes + value_place<DP>(r, piece) * 4);
            if (f != 0.0f) { x.x += f * o.x; x.y += f * o.y; x.z += f * o.z; x.w += f * o.w; }      /* 0: it may have left nothing */
        }
        *reinterpret_cast<float4 *>(part + r * DP + piece * 4) = x;
    }
}

/*
 * The items that begin in a CTA's teams and end in others, a query head per CTA, or two with half of the warps each where there
 * would be more CTAs than the GPU holds.  Items of up to kAlone parts have a warp each; at most one of a CTA's has more (it goes on
 * into other CTAs), and all warps of the head share its parts.  Lanes have four columns each.
 */
constexpr int kJoinWarps = 8, kJoinThreads = 32 * kJoinWarps, kAlone = 8;

/* A running join: values brought to the maximum so far.  A maximum of -infinity stands for nothing, whatever its values are. */
template <int DP> struct Joined {
    static constexpr int C = DP > 128 ? 2 : 1;
    float top = -INFINITY, sum = 0.0f, o[C][4] = {};
    template <int N> __device__ __forceinline__ void add(const float (&t)[N], const float (&s)[N], const float4 (&v)[N][C])
    {
        float now = top;
        bool nan = false;
#pragma unroll
        for (int k = 0; k < N; ++k) { now = fmaxf(now, t[k]); nan = nan || t[k] != t[k]; }
        const float ref = now == -INFINITY ? 0.0f : now, keep = exp2f(top - ref);
        top = now;
        sum = nan ? NAN : sum * keep;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][e] *= keep;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float f = exp2f(t[k] - ref);
            if (f == 0.0f) continue;
            sum += s[k] * f;
#pragma unroll
            for (int c = 0; c < C; ++c) { o[c][0] += v[k][c].x * f; o[c][1] += v[k][c].y * f; o[c][2] += v[k][c].z * f; o[c][3] += v[k][c].w * f; }
        }
    }
};

template <int DT, int DP>
__global__ void __launch_bounds__(kJoinThreads, 4) k_attend_join(const __grid_constant__ AttentionArgs a)
{
    using J = Joined<DP>;
    using T = typename Elem<DT>::type;
    __shared__ float s_top[kJoinWarps], s_sum[kJoinWarps];
    __shared__ __align__(16) float s_o[kJoinWarps][DP];
    grid_let_next_in();
    grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, warps = gridDim.y == a.rows ? kJoinWarps : kJoinWarps / 2, first = warp - warp % warps, nth = warp - first;
    const uint32_t r = blockIdx.y * (kJoinWarps / warps) + first / warps;
    const size_t part_floats = partial_floats(a.rows, DP);
    /* this warp's split, and the one that all share */
    const Split mine = nth < kTeams ? a.splits[blockIdx.x * kTeams + nth] : Split{0, 0, -1, 0, 0, 0, 0, 0};
    const Split last = a.splits[blockIdx.x * kTeams + kTeams - 1];
    Split big = last;
#pragma unroll
    for (int k = 0; k < kTeams - 1; ++k) {
        const Split s = a.splits[blockIdx.x * kTeams + k];
        if (s.first >= 0 && s.last - s.first + 1 > kAlone) big = s;
    }
    /* parts in their order: warps up to one0, a part per CTA up to one1, warps again */
    auto parts_of = [](const Split &s) { return min(s.one0, s.last + 1) - s.first + (s.one1 - s.one0) / kTeams + max(0, s.last + 1 - s.one1); };
    auto part_at = [&](const Split &s, int i) {
        const int before = min(s.one0, s.last + 1) - s.first, ones = (s.one1 - s.one0) / kTeams;
        const int w = i < before ? s.first + i : i < before + ones ? s.one0 + (i - before) * kTeams : s.one1 + (i - before - ones);
        return a.partial + ((size_t)w * 2 + (w == s.first ? s.slot : 0)) * part_floats;
    };
    auto there = [&](const Split &s) { return s.first >= 0 && r < min(a.rows, a.group - s.item % a.chunks * a.rows); };
    auto walk = [&](const Split &s, int i0, int i1, J &j) {
        constexpr int N = 4 / J::C;                               /* parts under way together */
        for (; i0 < i1; i0 += N) {
            float t[N], l[N];
            float4 v[N][J::C];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float *const p = part_at(s, min(i0 + k, i1 - 1));
                t[k] = i0 + k < i1 ? __ldcg(p + a.rows * DP + r) : -INFINITY;
                l[k] = __ldcg(p + a.rows * DP + a.rows + r);
#pragma unroll
                for (int c = 0; c < J::C; ++c)
                    if (DP >= 128 || lane < DP / 4) v[k][c] = __ldcg(reinterpret_cast<const float4 *>(p + r * DP + (lane + 32 * c) * 4));
            }
            j.add(t, l, v);
        }
    };
    auto finish = [&](const Split &s, const J &j) {
        const uint32_t head = s.item / a.chunks * a.group + s.item % a.chunks * a.rows + r;
        const float inv = j.sum == 0.0f ? 0.0f : 1.0f / j.sum;
        T *const out = reinterpret_cast<T *>(a.out + (size_t)s.sequence * a.ld_out) + (size_t)head * a.dim;
#pragma unroll
        for (int c = 0; c < J::C; ++c) {
            const float x[4] = {j.o[c][0] * inv, j.o[c][1] * inv, j.o[c][2] * inv, j.o[c][3] * inv};
            store_out<DT>(out, x, (lane + 32 * c) * 4, a.dim, a.out_vec);
        }
        if (a.lse && lane == 0) a.lse[(size_t)s.sequence * a.heads + head] = j.sum == 0.0f ? -INFINITY : (j.top + log2f(j.sum)) * kLn2;
    };

    if (there(mine) && parts_of(mine) <= kAlone) {
        J j;
        walk(mine, 0, parts_of(mine), j);
        finish(mine, j);
    }
    if (big.first < 0 || parts_of(big) <= kAlone) return;         /* the same for the whole CTA */
    const int n = there(big) ? parts_of(big) : 0;
    J j;
    walk(big, n * nth / warps, n * (nth + 1) / warps, j);
#pragma unroll
    for (int c = 0; c < J::C; ++c)
        if (DP >= 128 || lane < DP / 4) *reinterpret_cast<float4 *>(&s_o[warp][(lane + 32 * c) * 4]) = make_float4(j.o[c][0], j.o[c][1], j.o[c][2], j.o[c][3]);
    if (lane == 0) { s_top[warp] = top_of(j.top, j.sum); s_sum[warp] = j.sum; }
    __syncthreads();
    if (nth || !n) return;
    J total;
    constexpr int N = 4 / J::C;
    for (int w0 = first; w0 < first + warps; w0 += N) {
        float tops[N], l[N];
        float4 v[N][J::C];
#pragma unroll
        for (int w = 0; w < N; ++w) {
            tops[w] = s_top[w0 + w]; l[w] = s_sum[w0 + w];
#pragma unroll
            for (int c = 0; c < J::C; ++c)
                if (DP >= 128 || lane < DP / 4) v[w][c] = *reinterpret_cast<const float4 *>(&s_o[w0 + w][(lane + 32 * c) * 4]);
        }
        total.add(tops, l, v);
    }
    finish(big, total);
}

/* ------------------------------------------------------------------------ */
/* host                                                                      */
/* ------------------------------------------------------------------------ */
struct AttentionPlan { uint32_t rows, chunks, ctas; int dp; size_t split_bytes, bytes; };

template <int DT, int DP, int ROWS, bool VEC>
static cudaError_t launch_attend(const AttentionPlan &plan, cudaStream_t stream, const AttentionArgs &a)
{
    constexpr int shared = Shared<DT, DP, ROWS>::bytes;
    static_assert(shared <= 227 * 1024 - 1024, "rings");
    /* per device: an attribute of the kernel there */
    if (cudaError_t e = cudaFuncSetAttribute(k_attend<DT, DP, ROWS, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared)) return e;
    if (cudaError_t e = launch_op(k_attend<DT, DP, ROWS, VEC>, dim3(plan.ctas), dim3(32 * kTeams * team_warps<DT, ROWS>()), 1, shared, stream, a)) return e;
    return launch_op(k_attend_join<DT, DP>, dim3(plan.ctas, plan.ctas * plan.rows <= 4 * kSms ? plan.rows : (plan.rows + 1) / 2), dim3(kJoinThreads), 1, 0, stream, a);
}

template <int DT, int DP>
static cudaError_t launch_attend_d(bool vec, const AttentionPlan &plan, cudaStream_t stream, const AttentionArgs &a)
{
    if constexpr (DT == SIFAR_BF16) {
        if (plan.rows > 8) return vec ? launch_attend<DT, DP, 16, true>(plan, stream, a) : launch_attend<DT, DP, 16, false>(plan, stream, a);
    }
    if constexpr (DT == SIFAR_F32) {                              /* every head costs instructions, there or not: bound by them, not by memory */
        if (plan.rows <= 4) return vec ? launch_attend<DT, DP, 4, true>(plan, stream, a) : launch_attend<DT, DP, 4, false>(plan, stream, a);
    }
    return vec ? launch_attend<DT, DP, 8, true>(plan, stream, a) : launch_attend<DT, DP, 8, false>(plan, stream, a);
}

template <int DT>
static cudaError_t launch_attend_t(bool vec, const AttentionPlan &plan, cudaStream_t stream, const AttentionArgs &a)
{
    if (plan.dp == 64) return launch_attend_d<DT, 64>(vec, plan, stream, a);
    if (plan.dp == 128) return launch_attend_d<DT, 128>(vec, plan, stream, a);
    return launch_attend_d<DT, 256>(vec, plan, stream, a);
}

template <int DT> static int ctas_of(int dp, bool many)
{
    if constexpr (DT == SIFAR_BF16) {
        if (many) return dp == 64 ? ctas_per_sm<DT, 64, 16>() : dp == 128 ? ctas_per_sm<DT, 128, 16>() : ctas_per_sm<DT, 256, 16>();
    }
    return dp == 64 ? ctas_per_sm<DT, 64, 8>() : dp == 128 ? ctas_per_sm<DT, 128, 8>() : ctas_per_sm<DT, 256, 8>();
}

static int plan_attention(const char *fn, const sifar_decode_attention_args *g, CacheShape &c, AttentionPlan &p)
{
    if (!g) { set_error("%s: no argument block", fn); return SIFAR_ERR_INVALID; }
    if (int rc = check_cache(fn, c, g->dtype, g->kv_heads, g->head_dim, g->pages, g->page_size, g->max_pages, g->sequences, g->ld_page_table,
                             g->stride_page, g->stride_token, g->stride_head)) return rc;
    if (g->heads < 1 || g->heads % g->kv_heads || (size_t)g->heads * c.dim >= (1u << 20) || !std::isfinite(g->scale)) {
        set_error("%s: need heads that kv_heads divides, heads * head_dim below 2^20 and a finite scale", fn);
        return SIFAR_ERR_INVALID;
    }
    const bool bf16 = g->dtype == SIFAR_BF16;
    const uint32_t group = (uint32_t)(g->heads / g->kv_heads), most = bf16 ? 16u : 8u;
    p.chunks = (group + most - 1) / most;
    p.rows = (group + p.chunks - 1) / p.chunks;
    p.dp = c.dim <= 64 ? 64 : c.dim <= 128 ? 128 : 256;
    p.ctas = kSms * (unsigned)(bf16 ? ctas_of<SIFAR_BF16>(p.dp, p.rows > 8) : ctas_of<SIFAR_F32>(p.dp, false));
    p.split_bytes = (size_t)p.ctas * kTeams * sizeof(Split);
    p.bytes = p.split_bytes + (size_t)p.ctas * kTeams * 2 * partial_floats(p.rows, p.dp) * sizeof(float);
    p.bytes = (p.bytes + 15) / 16 * 16;
    return SIFAR_OK;
}

}  /* namespace sifar */

using namespace sifar;

extern "C" size_t sifar_decode_attention_workspace(const sifar_decode_attention_args *g)
{
    CacheShape c;
    AttentionPlan p;
    return plan_attention("sifar_decode_attention_workspace", g, c, p) == SIFAR_OK ? p.bytes : 0;
}

extern "C" int sifar_decode_attention(const sifar_decode_attention_args *g, void *stream)
{
    static const char *fn = "sifar_decode_attention";
    CacheShape c;
    AttentionPlan p;
    if (int rc = plan_attention(fn, g, c, p)) return rc;
    if (g->sequences == 0) return SIFAR_OK;
    if (!g->q || !g->k_cache || !g->v_cache || !g->lengths || !g->out || (!g->page_table && c.max_pages)) {
        set_error("%s: q, the caches, page_table, lengths and out are needed", fn);
        return SIFAR_ERR_INVALID;
    }
    if (!g->workspace || (uintptr_t)g->workspace % 16 || g->workspace_bytes < p.bytes) {
        set_error("%s: needs %zu bytes of workspace on a 16-byte boundary", fn, p.bytes);
        return SIFAR_ERR_INVALID;
    }
    const size_t es = c.es, S = g->sequences, cols = (size_t)g->heads * c.dim, lses = S * (size_t)g->heads;
    const size_t entries = (S - 1) * c.ld_table + c.max_pages;
    const RowArray all[] = {
        RowArray{"q", g->q, S, cols, g->ld_q ? g->ld_q : cols, es, false},
        RowArray{"page_table", g->page_table, 1, entries, entries, sizeof(int), false},
        RowArray{"lengths", g->lengths, 1, S, S, sizeof(int), false},
        RowArray{"out", g->out, S, cols, g->ld_out ? g->ld_out : cols, es, true},
        RowArray{"lse", g->lse, 1, lses, lses, sizeof(float), true},
        RowArray{"workspace", g->workspace, 1, p.bytes, p.bytes, 1, true},
    };
    if (int rc = check_arrays(fn, all, 6)) return rc;
    const size_t extent = cache_extent(c);
    const RowArray kc{"k_cache", g->k_cache, 1, 1, 1, es, false}, vc{"v_cache", g->v_cache, 1, 1, 1, es, false};
    if (int rc = check_array(fn, kc)) return rc;
    if (int rc = check_array(fn, vc)) return rc;
    for (const RowArray &x : all)
        if (x.out && (touches(x, g->k_cache, extent) || touches(x, g->v_cache, extent))) { set_error("%s: %s overlaps the cache", fn, x.name); return SIFAR_ERR_INVALID; }

    AttentionArgs a;
    a.q = (const char *)g->q; a.k = (const char *)g->k_cache; a.v = (const char *)g->v_cache;
    a.out = (char *)g->out; a.lse = g->lse; a.lengths = g->lengths;
    a.pages = device_pages(c, g->page_table);
    a.splits = (Split *)g->workspace;
    a.partial = (float *)((char *)g->workspace + p.split_bytes);
    a.ld_q = all[0].ld * es; a.ld_out = all[3].ld * es;
    a.sequences = (uint32_t)S;
    a.window = g->window >= ((size_t)1 << 31) ? 0u : (uint32_t)g->window;
    a.limit = (uint32_t)(c.max_pages * c.page_size);
    a.heads = (uint32_t)g->heads; a.kv_heads = (uint32_t)g->kv_heads; a.group = a.heads / a.kv_heads;
    a.chunks = p.chunks; a.rows = p.rows; a.dim = (uint32_t)c.dim;
    a.scale = g->scale * kLog2e;
    a.q_vec = rows_aligned16(all[0]) && c.dim * es % 16 == 0;
    a.out_vec = (uintptr_t)g->out % (4 * es) == 0 && c.dim % 4 == 0 && (S == 1 || all[3].ld % 4 == 0);
    const bool vec = cache_aligned16(c, g->k_cache, g->v_cache) && c.dim * es % 16 == 0;
    const cudaError_t err = g->dtype == SIFAR_BF16 ? launch_attend_t<SIFAR_BF16>(vec, p, (cudaStream_t)stream, a)
                                                   : launch_attend_t<SIFAR_F32>(vec, p, (cudaStream_t)stream, a);
    SIFAR_CUDA(err);
    return SIFAR_OK;
}
