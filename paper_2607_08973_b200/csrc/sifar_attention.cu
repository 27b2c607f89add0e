/*
 * sifar_attention.cu - attention of one new token per sequence over a paged cache, split over the cache's length.
 *
 * An item is a key head of a sequence with up to 16 (binary32: 8) of the query heads that read it.  All items' tiles of
 * 64 tokens in a row are cut into equal shares, one per CTA, whatever the lengths; an item that ends up with several CTAs is
 * put together by a second kernel from their maxima, sums and weighted values.
 *
 * A warp takes 16 tokens at a time (a strip) through a ring of its own in shared memory, filled by asynchronous
 * 16-byte copies two strips ahead; warps of a CTA meet only when an item is done.
 */
#include "sifar_cache.cuh"
#include "sifar_norm_shape.cuh"

namespace sifar {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kTile = 64;                    /* tokens; what the shares are counted in */
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

/* Where a split item lies in the workspace: partials of CTAs first .. last, in the order of the tokens. */
struct Split { int sequence, kv_head, chunk, first, last, slot, pad[2]; };       /* slot of `first`'s partial; first < 0: none */

struct AttentionArgs {
    const char *q, *k, *v;
    char *out;
    float *lse;
    const int *lengths;
    Pages pages;
    Split *splits;                           /* one per CTA */
    float *partial;                          /* CTA x 2 partials */
    unsigned long long ld_q, ld_out;         /* bytes */
    uint32_t sequences, window, limit;       /* limit = max_pages * page_size */
    uint32_t heads, kv_heads, group, chunks, rows, dim;   /* rows = query heads of an item, chunks of them per key head */
    float scale;                             /* times log2(e) */
};

/* Floats of a partial: rows x dim_pad values, rows maxima, rows sums; the next one starts on 16 bytes again. */
__host__ __device__ __forceinline__ size_t partial_floats(uint32_t rows, int dim_pad) { return ((size_t)rows * (dim_pad + 2) + 3) / 4 * 4; }

/* First visible token and the one behind the last. */
__device__ __forceinline__ void visible(const AttentionArgs &a, uint32_t s, uint32_t &lo, uint32_t &hi)
{
    hi = (uint32_t)min(max(a.lengths[s], 0), (int)a.limit);
    lo = a.window && hi > a.window ? hi - a.window : 0u;
}
__device__ __forceinline__ uint32_t tiles_of(const AttentionArgs &a, uint32_t s)
{
    uint32_t lo, hi;
    visible(a, s, lo, hi);
    return max(1u, (hi - lo + kTile - 1) / kTile);       /* an empty sequence has an item too: its zeros */
}

/* Tile number `at` in the row of all items' tiles: which sequence, and how many of its items' tiles lie before. */
struct Place { unsigned long long total, begin, end; uint32_t sequence; unsigned long long before; };

/*
 * The share of this CTA and the sequence that it begins in.  Every thread adds up the tiles of a run of sequences; the
 * one whose run holds the share's begin walks it.
 */
__device__ __forceinline__ Place find_share(const AttentionArgs &a, unsigned long long *s_sum, Place *s_place)
{
    const uint32_t run = (a.sequences + kThreads - 1) / kThreads, s0 = threadIdx.x * run, s1 = min(a.sequences, s0 + run);
    const unsigned long long items = (unsigned long long)a.kv_heads * a.chunks;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    unsigned long long mine = 0;
    for (uint32_t s = s0; s < s1; ++s) mine += tiles_of(a, s);
    mine *= items;
    unsigned long long sum = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(0xFFFFFFFFu, sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 31) s_sum[warp] = sum;
    __syncthreads();
    unsigned long long before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    before += sum - mine;
    const unsigned long long share = (total + gridDim.x - 1) / gridDim.x, begin = min(total, share * blockIdx.x), end = min(total, begin + share);
    if (begin < end && begin >= before && begin < before + mine) {
        Place p{total, begin, end, s0, before};
        for (; p.sequence < s1; ++p.sequence) {
            const unsigned long long t = tiles_of(a, p.sequence) * items;
            if (begin < p.before + t) break;
            p.before += t;
        }
        *s_place = p;
    }
    __syncthreads();
    return begin < end ? *s_place : Place{total, begin, end, 0, 0};
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
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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

/* Issues the copies of the strip from token t0 on.  `offset` is that of token t0 + (lane % tokens), -1 if it is masked. */
template <int DT, int DP, bool VEC>
__device__ __forceinline__ void fetch(const AttentionArgs &a, char *ring, int stage, long long offset, unsigned long long head)
{
    using R = Ring<DT, DP>;
    const int lane = threadIdx.x & 31;
    char *const ks = ring + stage * 2 * R::strip, *const vs = ks + R::strip;
    if (VEC) {
        /* R::chunks lanes per row */
        constexpr int rows = 32 / R::chunks > 0 ? 32 / R::chunks : 1, per = R::chunks > 32 ? R::chunks / 32 : 1;
#pragma unroll
        for (int r0 = 0; r0 < R::tokens; r0 += rows) {
            const int r = r0 + (R::chunks >= 32 ? 0 : lane / R::chunks);
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
        for (int r = 0; r < R::tokens; ++r) {
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

/* ------------------------------------------------------------------------ */
/* what a warp holds of an item                                              */
/* ------------------------------------------------------------------------ */
/*
 * bf16: matrix instructions of 16 rows (query heads) x 16 x 8.  Up to eight heads (ROWS = 8) take the upper half of the
 * rows, and the probabilities go in as two bf16 values, the rounded one above and what it leaves below: they keep 16 bits
 * at no further instruction.  With 16 heads that takes a second product.
 */
template <int DP, int ROWS> struct StateBf16 {
    using R = Ring<SIFAR_BF16, DP>;
    static constexpr int H = ROWS / 8;
    uint32_t q[DP / 16][2 * H];
    float o[DP / 8][4];
    float m[H], l[H];                               /* l: this lane's columns */

    __device__ __forceinline__ void begin(const AttentionArgs &a, const char *q_row, uint32_t rows, const float *)
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            m[h] = -INFINITY; l[h] = 0.0f;
            const uint32_t row = g + 8 * h;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint32_t d = i * 16 + x * 8 + 2 * j;
                    const uint16_t *p = reinterpret_cast<const uint16_t *>(q_row) + row * a.dim + d;
                    uint32_t w = 0;
                    if (row < rows && d < a.dim) w = p[0];
                    if (row < rows && d + 1 < a.dim) w |= (uint32_t)p[1] << 16;
                    q[i][x * H + h] = w;
                }
        }
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    }

    /* seen: bit t set where token t of the strip counts */
    __device__ __forceinline__ void strip(const AttentionArgs &a, const char *ring, int stage, uint32_t seen, float *)
    {
        const int lane = threadIdx.x & 31, j = lane & 3;
        const uint32_t ks = shared_at(ring + stage * 2 * R::strip), vs = ks + R::strip;
        float s[2][4] = {};
        {
            const int row = (lane & 7) + ((lane >> 4) & 1) * 8, half = (lane >> 3) & 1;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                uint32_t b[4];
                load_matrices(b, ks + row * R::row + R::place(row, 2 * i + half) * 16);
                if (H == 1) {
                    multiply(s[0], q[i][0], 0u, q[i][1], 0u, b[0], b[1]);
                    multiply(s[1], q[i][0], 0u, q[i][1], 0u, b[2], b[3]);
                } else {
                    multiply(s[0], q[i][0], q[i][H - 1], q[i][H], q[i][2 * H - 1], b[0], b[1]);
                    multiply(s[1], q[i][0], q[i][H - 1], q[i][H], q[i][2 * H - 1], b[2], b[3]);
                }
            }
        }
        float keep[H];
        uint32_t p[H][2], rest[H][2];
#pragma unroll
        for (int h = 0; h < H; ++h) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = seen >> ((i >> 1) * 8 + 2 * j + (i & 1)) & 1u;
                x[i] = in ? s[i >> 1][2 * h + (i & 1)] * a.scale : -INFINITY;
            }
            float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const float now = fmaxf(m[h], top), ref = now == -INFINITY ? 0.0f : now;
            keep[h] = exp2f(m[h] - ref);
            m[h] = now;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = exp2f(x[i] - ref);
            l[h] = l[h] * keep[h] + ((x[0] + x[1]) + (x[2] + x[3]));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                p[h][i] = pair_bf16(x[2 * i], x[2 * i + 1]);
                rest[h][i] = rest_bf16(x[2 * i], x[2 * i + 1], p[h][i]);
            }
        }
        bool moved = keep[0] != 1.0f;
        if (H == 2) moved = moved || keep[H - 1] != 1.0f;
        if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) {
                o[i][0] *= keep[0]; o[i][1] *= keep[0];
                o[i][2] *= keep[H - 1]; o[i][3] *= keep[H - 1];
            }
        }
        const int row = lane & 15, half = lane >> 4;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            uint32_t b[4];
            load_matrices_turned(b, vs + row * R::row + R::place(row, 2 * i + half) * 16);
            if (H == 1) {
                multiply(o[2 * i], p[0][0], rest[0][0], p[0][1], rest[0][1], b[0], b[1]);
                multiply(o[2 * i + 1], p[0][0], rest[0][0], p[0][1], rest[0][1], b[2], b[3]);
            } else {
                multiply(o[2 * i], p[0][0], p[H - 1][0], p[0][1], p[H - 1][1], b[0], b[1]);
                multiply(o[2 * i + 1], p[0][0], p[H - 1][0], p[0][1], p[H - 1][1], b[2], b[3]);
                multiply(o[2 * i], rest[0][0], rest[H - 1][0], rest[0][1], rest[H - 1][1], b[0], b[1]);
                multiply(o[2 * i + 1], rest[0][0], rest[H - 1][0], rest[0][1], rest[H - 1][1], b[2], b[3]);
            }
        }
    }

    /* The warp's part of the item: `values` rows x DP, then ROWS maxima, ROWS sums. */
    __device__ __forceinline__ void leave(float *values, float *top, float *sum)
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            float t = l[h];
            t += __shfl_xor_sync(0xFFFFFFFFu, t, 1);
            t += __shfl_xor_sync(0xFFFFFFFFu, t, 2);
            if (j == 0) { top[g + 8 * h] = m[h]; sum[g + 8 * h] = t; }
        }
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
            float2 *to = reinterpret_cast<float2 *>(values + g * DP + i * 8 + 2 * j);
            if (H == 1) *to = make_float2(o[i][0] + o[i][2], o[i][1] + o[i][3]);
            else {
                *to = make_float2(o[i][0], o[i][1]);
                to[4 * DP] = make_float2(o[i][2], o[i][3]);
            }
        }
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

    __device__ __forceinline__ void begin(const AttentionArgs &, const char *, uint32_t, const float *q_shared)
    {
        q = q_shared;
#pragma unroll
        for (int h = 0; h < ROWS; ++h) {
            m[h] = -INFINITY; l[h] = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c) o[h][c][0] = o[h][c][1] = o[h][c][2] = o[h][c][3] = 0.0f;
        }
    }

    __device__ __forceinline__ void strip(const AttentionArgs &a, const char *ring, int stage, uint32_t seen, float *p_shared)
    {
        const int lane = threadIdx.x & 31, t = lane / L, part = lane % L;
        const char *const ks = ring + stage * 2 * R::strip, *const vs = ks + R::strip;
        float s[ROWS] = {};
#pragma unroll 4
        for (int i = part; i < R::chunks; i += L) {
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

    __device__ __forceinline__ void leave(float *values, float *top, float *sum)
    {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int h = 0; h < ROWS; ++h) {
            const float t = warp_sum(l[h]);
            if (lane == 0) { top[h] = m[h]; sum[h] = t; }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float4 x = make_float4(o[h][c][0], o[h][c][1], o[h][c][2], o[h][c][3]);
                if (half == 2) {
                    x.x += __shfl_xor_sync(0xFFFFFFFFu, x.x, 16); x.y += __shfl_xor_sync(0xFFFFFFFFu, x.y, 16);
                    x.z += __shfl_xor_sync(0xFFFFFFFFu, x.z, 16); x.w += __shfl_xor_sync(0xFFFFFFFFu, x.w, 16);
                }
                if (half == 1 || lane < 16)
                    *reinterpret_cast<float4 *>(values + h * DP + (half == 2 ? lane & 15 : lane + 32 * c) * 4) = x;
            }
        }
    }
};

template <int DT, int DP, int ROWS> struct StateOf { using type = StateBf16<DP, ROWS>; };
template <int DP, int ROWS> struct StateOf<SIFAR_F32, DP, ROWS> { using type = StateF32<DP, ROWS>; };

/* Shared memory: the rings, later the warps' parts in their place; behind them binary32 queries and probabilities. */
template <int DT, int DP, int ROWS> struct Shared {
    static constexpr int rings = kWarps * Ring<DT, DP>::bytes, parts = kWarps * ROWS * (DP + 2) * 4;
    static constexpr int queries = rings > parts ? rings : parts;
    static constexpr int bytes = queries + (DT == SIFAR_F32 ? (ROWS * DP + kWarps * ROWS * Ring<DT, DP>::tokens) * 4 : 0);
};

template <int DT, int DP, int ROWS, bool VEC>
__global__ void __launch_bounds__(kThreads) k_attend(const __grid_constant__ AttentionArgs a)
{
    using R = Ring<DT, DP>;
    extern __shared__ __align__(128) char smem[];
    __shared__ unsigned long long s_sum[kWarps];
    __shared__ Place s_place;
    __shared__ float s_w[kWarps][ROWS], s_m[ROWS], s_l[ROWS];
    constexpr int es = DT == SIFAR_BF16 ? 2 : 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    char *const ring = smem + warp * R::bytes;
    float *const parts = reinterpret_cast<float *>(smem);                           /* warp x ROWS x DP, maxima, sums */
    float *const tops = parts + kWarps * ROWS * DP, *const sums = tops + kWarps * ROWS;
    float *const q_shared = reinterpret_cast<float *>(smem + Shared<DT, DP, ROWS>::queries);
    float *const p_shared = q_shared + ROWS * DP + warp * ROWS * R::tokens;
    grid_let_next_in();
    grid_wait();

    const Place place = find_share(a, s_sum, &s_place);
    if (threadIdx.x == 0) a.splits[blockIdx.x].first = -1;
    unsigned long long at = place.begin, before = place.before;
    uint32_t sequence = place.sequence;
    const unsigned long long share = (place.total + gridDim.x - 1) / gridDim.x;
    const size_t part_floats = partial_floats(a.rows, DP);

    while (at < place.end) {
        /* the item that tile `at` belongs to */
        const uint32_t tiles = tiles_of(a, sequence);
        const uint32_t item = (uint32_t)((at - before) / tiles), kv_head = item / a.chunks, chunk = item % a.chunks;
        const unsigned long long item_begin = before + (unsigned long long)item * tiles, item_end = item_begin + tiles;
        const uint32_t tile0 = (uint32_t)(at - item_begin), tile1 = (uint32_t)(min(item_end, place.end) - item_begin);
        uint32_t lo, hi;
        visible(a, sequence, lo, hi);
        const uint32_t end = min(hi, lo + tile1 * kTile), begin = lo + tile0 * kTile;
        const uint32_t rows = min(a.rows, a.group - chunk * a.rows), head = kv_head * a.group + chunk * a.rows;
        const char *const q_row = a.q + sequence * a.ld_q + (size_t)head * a.dim * es;
        const int *const table = a.pages.table + sequence * a.pages.ld_table;
        const unsigned long long head_at = kv_head * a.pages.stride_head;

        if (DT == SIFAR_F32) {
            for (uint32_t i = threadIdx.x; i < ROWS * DP; i += kThreads) {
                const uint32_t r = i / DP, d = i % DP;
                q_shared[i] = r < rows && d < a.dim ? reinterpret_cast<const float *>(q_row)[r * a.dim + d] : 0.0f;
            }
            __syncthreads();
        }
        typename StateOf<DT, DP, ROWS>::type state;

        /* this warp's strips: begin + (warp + i * kWarps) * tokens */
        const uint32_t strips = end > begin ? (end - begin + R::tokens - 1) / R::tokens : 0u;
        const uint32_t mine = strips > (uint32_t)warp ? (strips - warp + kWarps - 1) / kWarps : 0u;
        auto offset_of = [&](uint32_t i) -> long long {
            const uint32_t t = begin + (warp + i * kWarps) * R::tokens + lane % R::tokens;
            return i < mine && t < end ? token_offset(a.pages, table, t) : -1ll;
        };
        uint32_t seen[R::stages];
        /* strips 0 .. stages - 2 are under way before the first is used */
        long long next = offset_of(0);
#pragma unroll
        for (int i = 0; i < R::stages - 1; ++i) {
            const long long now = next;
            next = offset_of(i + 1);
            seen[i] = __ballot_sync(0xFFFFFFFFu, now >= 0);
            if ((uint32_t)i < mine) fetch<DT, DP, VEC>(a, ring, i, now, head_at);
            copies_commit();
        }
        state.begin(a, q_row, rows, q_shared);
        for (uint32_t i0 = 0; i0 < mine; i0 += R::stages) {
#pragma unroll
            for (int u = 0; u < R::stages; ++u) {
                const uint32_t i = i0 + u;
                if (i >= mine) break;
                constexpr int last = R::stages - 1;
                const int to = (u + last) % R::stages;
                const long long now = next;
                next = offset_of(i + R::stages);
                copies_wait<R::stages - 2>();
                __syncwarp();
                seen[to] = __ballot_sync(0xFFFFFFFFu, now >= 0);
                if (i + last < mine) fetch<DT, DP, VEC>(a, ring, to, now, head_at);
                copies_commit();
                state.strip(a, ring, u, seen[u], p_shared);
            }
        }
        copies_wait<0>();
        __syncthreads();                                          /* the rings become the warps' parts */
        state.leave(parts + warp * ROWS * DP, tops + warp * ROWS, sums + warp * ROWS);
        __syncthreads();
        if (threadIdx.x < ROWS) {
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, tops[w * ROWS + threadIdx.x]);
            const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = exp2f(tops[w * ROWS + threadIdx.x] - ref);
                s_w[w][threadIdx.x] = f;
                sum += f * sums[w * ROWS + threadIdx.x];
            }
            s_m[threadIdx.x] = top; s_l[threadIdx.x] = sum;
        }
        __syncthreads();
        const bool whole = tile0 == 0 && tile1 == tiles;
        /* slot 0: the item that the share begins in; slot 1: one that it leaves unfinished */
        const int slot = item_begin <= place.begin ? 0 : 1;
        float *const part = a.partial + ((size_t)blockIdx.x * 2 + slot) * part_floats;
        for (uint32_t i = threadIdx.x; i < rows * (DP / 4); i += kThreads) {
            const uint32_t r = i / (DP / 4), d = i % (DP / 4) * 4;
            float x[4] = {};
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = s_w[w][r];
                const float4 o = *reinterpret_cast<const float4 *>(parts + (w * ROWS + r) * DP + d);
                x[0] += f * o.x; x[1] += f * o.y; x[2] += f * o.z; x[3] += f * o.w;
            }
            if (whole) {
                const float sum = s_l[r], inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                auto *out = reinterpret_cast<typename Elem<DT>::type *>(a.out + sequence * a.ld_out) + (size_t)(head + r) * a.dim + d;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e < a.dim) out[e] = narrow<DT>(x[e] * inv);
            } else {
                *reinterpret_cast<float4 *>(part + r * DP + d) = make_float4(x[0], x[1], x[2], x[3]);
            }
        }
        if (threadIdx.x < rows) {
            const float top = s_m[threadIdx.x], sum = s_l[threadIdx.x];
            if (whole) {
                if (a.lse) a.lse[sequence * (size_t)a.heads + head + threadIdx.x] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
            } else {
                part[a.rows * DP + threadIdx.x] = top;
                part[a.rows * DP + a.rows + threadIdx.x] = sum;
            }
        }
        if (!whole && threadIdx.x == 0 && tile0 == 0) {
            Split s{(int)sequence, (int)kv_head, (int)chunk, (int)blockIdx.x, (int)((item_end - 1) / share), slot, {0, 0}};
            a.splits[blockIdx.x] = s;
        }
        __syncthreads();                                          /* before the rings are filled again */
        at = item_begin + tile1;
        if (at == before + (unsigned long long)a.kv_heads * a.chunks * tiles) { before = at; ++sequence; }
    }
}

/*
 * An item whose tiles several CTAs had: one CTA per query head.  Warps take partials in turn, each lane four (eight) columns.
 */
constexpr int kJoinWarps = 8;
template <int DT, int DP>
__global__ void __launch_bounds__(32 * kJoinWarps) k_attend_join(const __grid_constant__ AttentionArgs a)
{
    __shared__ float s_top[kJoinWarps], s_sum[kJoinWarps];
    __shared__ __align__(16) float s_o[kJoinWarps][DP];
    grid_let_next_in();
    grid_wait();
    const Split s = a.splits[blockIdx.x];
    const uint32_t r = blockIdx.y;
    if (s.first < 0 || r >= min(a.rows, a.group - s.chunk * a.rows)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const size_t part_floats = partial_floats(a.rows, DP);
    const int n = s.last - s.first + 1;
    auto part = [&](int i) { return a.partial + ((size_t)(s.first + i) * 2 + (i == 0 ? s.slot : 0)) * part_floats; };
    /* the largest maximum, then the sum with every part brought to it */
    float top = -INFINITY;
    for (int i = threadIdx.x; i < n; i += 32 * kJoinWarps) top = fmaxf(top, part(i)[a.rows * DP + r]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, s_top[w]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, o[DP / 32] = {};
#pragma unroll 4
    for (int i = warp; i < n; i += kJoinWarps) {
        const float *p = part(i);
        const float f = exp2f(p[a.rows * DP + r] - ref);
        sum += f * p[a.rows * DP + a.rows + r];
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) o[c] += f * p[r * DP + c * 32 + lane];
    }
#pragma unroll
    for (int c = 0; c < DP / 32; ++c) s_o[warp][c * 32 + lane] = o[c];
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) sum += s_sum[w];
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const uint32_t head = s.kv_head * a.group + s.chunk * a.rows + r;
    for (uint32_t d = threadIdx.x; d < a.dim; d += 32 * kJoinWarps) {
        float x = 0.0f;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) x += s_o[w][d];
        reinterpret_cast<typename Elem<DT>::type *>(a.out + (size_t)s.sequence * a.ld_out)[(size_t)head * a.dim + d] = narrow<DT>(x * inv);
    }
    if (a.lse && threadIdx.x == 0) a.lse[(size_t)s.sequence * a.heads + head] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

/* ------------------------------------------------------------------------ */
/* host                                                                      */
/* ------------------------------------------------------------------------ */
struct AttentionPlan { uint32_t rows, chunks, ctas; int dp; size_t split_bytes, bytes; };

/* CTAs that an SM holds by shared memory (227 KB, 1 KB of it per CTA for the system). */
constexpr int ctas_per_sm(int shared) { return 227 * 1024 / (shared + 1024) < 8 ? 227 * 1024 / (shared + 1024) : 8; }

template <int DT, int DP, int ROWS, bool VEC>
static cudaError_t launch_attend(const AttentionPlan &plan, cudaStream_t stream, const AttentionArgs &a)
{
    constexpr int shared = Shared<DT, DP, ROWS>::bytes;
    static_assert(shared <= 227 * 1024 - 1024, "rings");
    /* per device: an attribute of the kernel there */
    if (cudaError_t e = cudaFuncSetAttribute(k_attend<DT, DP, ROWS, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared)) return e;
    if (cudaError_t e = launch_op(k_attend<DT, DP, ROWS, VEC>, dim3(plan.ctas), dim3(kThreads), 1, shared, stream, a)) return e;
    return launch_op(k_attend_join<DT, DP>, dim3(plan.ctas, plan.rows), dim3(32 * kJoinWarps), 1, 0, stream, a);
}

template <int DT, int DP>
static cudaError_t launch_attend_d(bool vec, const AttentionPlan &plan, cudaStream_t stream, const AttentionArgs &a)
{
    if constexpr (DT == SIFAR_BF16) {
        if (plan.rows > 8) return vec ? launch_attend<DT, DP, 16, true>(plan, stream, a) : launch_attend<DT, DP, 16, false>(plan, stream, a);
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

template <int DT> static int shared_of(int dp, bool many)
{
    if constexpr (DT == SIFAR_BF16) {
        if (many) return dp == 64 ? Shared<DT, 64, 16>::bytes : dp == 128 ? Shared<DT, 128, 16>::bytes : Shared<DT, 256, 16>::bytes;
    }
    return dp == 64 ? Shared<DT, 64, 8>::bytes : dp == 128 ? Shared<DT, 128, 8>::bytes : Shared<DT, 256, 8>::bytes;
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
    p.ctas = kSms * (unsigned)ctas_per_sm(bf16 ? shared_of<SIFAR_BF16>(p.dp, p.rows > 8) : shared_of<SIFAR_F32>(p.dp, false));
    p.split_bytes = p.ctas * sizeof(Split);
    p.bytes = p.split_bytes + (size_t)p.ctas * 2 * partial_floats(p.rows, p.dp) * sizeof(float);
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
    const bool vec = cache_aligned16(c, g->k_cache, g->v_cache) && c.dim * es % 16 == 0;
    const cudaError_t err = g->dtype == SIFAR_BF16 ? launch_attend_t<SIFAR_BF16>(vec, p, (cudaStream_t)stream, a)
                                                   : launch_attend_t<SIFAR_F32>(vec, p, (cudaStream_t)stream, a);
    SIFAR_CUDA(err);
    return SIFAR_OK;
}
