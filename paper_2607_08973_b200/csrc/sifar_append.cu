/*
 * sifar_append.cu - new tokens' queries and keys turned by their positions, keys and values into the paged cache.
 *
 * A CTA per token: cosines and sines of the token's angles once, in shared memory, for all its heads.  A thread has the same
 * place in every head that it takes; its first loads, into shared memory, are under way while it is looked up where the token
 * belongs and the angles are computed.  Bound by memory, every element is read and written once, and by instructions.  8192 tokens of
 * 32 + 8 + 8 bf16 heads of 128 take 38 us, 5.3 TB/s, 79 % of the issue slots (without the loads ahead, a thread's place worked out for
 * each head: 46); one token 3.2 us, the launch.
 */
#include "sifar_cache.cuh"
#include "sifar_norm_shape.cuh"

namespace sifar {

struct AppendArgs {
    const char *q, *k, *v;
    char *q_out, *k_cache, *v_cache;
    const int *sequence, *position;
    const float *inv_freq;
    Pages pages;
    unsigned long long ld_q, ld_k, ld_v, ld_q_out;     /* bytes */
    uint32_t sequences;
    uint32_t heads, kv_heads, dim, half;               /* half = rotary_dim / 2 */
    uint32_t turned, copied;                           /* items of a head that turns, of one that is copied */
};

/* V elements from one place on, as binary32 or as they are. */
template <int DT, int V> struct Piece {
    using T = typename Elem<DT>::type;
    uint32_t w[V == 1 ? 1 : 4];
    __device__ __forceinline__ void load(const char *p)
    {
        if (V == 1) w[0] = *reinterpret_cast<const T *>(p);
        else *reinterpret_cast<uint4 *>(w) = *reinterpret_cast<const uint4 *>(p);
    }
    __device__ __forceinline__ void load_shared(const uint4 *p) { *reinterpret_cast<uint4 *>(w) = *p; }
    __device__ __forceinline__ void store(char *p) const
    {
        if (V == 1) *reinterpret_cast<T *>(p) = (T)w[0];
        else *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(w);
    }
    __device__ __forceinline__ float get(int i) const
    {
        if (DT == SIFAR_F32) return __uint_as_float(w[i]);
        if (V == 1) return __uint_as_float(w[0] << 16);
        return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void set(int i, float f)
    {
        if (DT == SIFAR_F32) w[i] = __float_as_uint(f);
        else if (V == 1) w[0] = narrow<DT>(f);
        else w[i / 2] = i & 1 ? (w[i / 2] & 0xFFFFu) | (uint32_t)narrow<DT>(f) << 16 : (w[i / 2] & 0xFFFF0000u) | narrow<DT>(f);
    }
};

__device__ __forceinline__ void copy16(uint4 *to, const char *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

/*
 * An item is what a thread loads, turns and stores at once: V pairs in two pieces (halves apart), V / 2 pairs in one
 * piece (interleaved; V = 1: one pair in two pieces), or a piece that is copied.
 */
template <int DT, int V, bool INTER>
__global__ void __launch_bounds__(512, 3) k_append(const __grid_constant__ AppendArgs a)
{
    constexpr int es = DT == SIFAR_BF16 ? 2 : 4, B = 2;
    constexpr bool kOne = INTER && V > 1;              /* a pair lies within a piece */
    constexpr int n = kOne ? V / 2 : V;                /* pairs of an item */
    extern __shared__ uint4 s_item[];                  /* whole pieces: a thread's first items, [piece][thread] */
    __shared__ __align__(16) float s_cos[SIFAR_CACHE_MAX_HEAD_DIM / 2], s_sin[SIFAR_CACHE_MAX_HEAD_DIM / 2];
    const uint32_t token = blockIdx.x;
    grid_let_next_in();
    grid_wait();
    const int position = a.position[token];
    const uint32_t sequence = a.sequence ? (uint32_t)a.sequence[token] : token;
    /* the thread's item of a head, and the first and the next of its heads */
    const uint32_t pairs = kOne ? 2 * a.half / V : a.half / V;       /* items of a head that have pairs */
    const uint32_t first = threadIdx.x / a.turned, i = threadIdx.x - first * a.turned, step = blockDim.x / a.turned;
    const bool turn = i < pairs;
    const uint32_t x = turn ? (kOne ? i * V : INTER ? 2 * i : i * V) : 2 * a.half + (i - pairs) * V;     /* elements of the head */
    const uint32_t y = x + (INTER ? 1u : a.half);                    /* the second piece: of pairs in two */
    const bool two = turn && !kOne;
    const uint32_t heads = first < step ? a.heads + a.kv_heads : 0u;
    const char *const q = a.q + token * a.ld_q, *const k = a.k + token * a.ld_k;
    char *const q_out = a.q_out + token * a.ld_q_out;
    auto source = [&](uint32_t h) { return h < a.heads ? q + (size_t)h * a.dim * es : k + (size_t)(h - a.heads) * a.dim * es; };
    /* the first loads go out before it is known where the token belongs */
    const uint32_t vfirst = threadIdx.x / a.copied, vi = threadIdx.x - vfirst * a.copied, vstep = blockDim.x / a.copied, values = vfirst < vstep ? a.kv_heads : 0u;
    const char *const v = a.v + token * a.ld_v + vi * V * es;
    auto slot = [&](int i) { return s_item + i * blockDim.x + threadIdx.x; };
    if constexpr (V > 1) {
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const uint32_t h = first + b * step;
            if (h >= heads) break;
            copy16(slot(2 * b), source(h) + x * es);
            if (two) copy16(slot(2 * b + 1), source(h) + y * es);
        }
        if (vfirst < values) copy16(slot(2 * B), v + (size_t)vfirst * a.dim * es);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (position < 0 || sequence >= a.sequences) {
        if constexpr (V > 1) asm volatile("cp.async.wait_group 0;" ::: "memory");        /* nothing may arrive in a CTA that is gone */
        return;
    }
    const long long at = token_offset(a.pages, a.pages.table + sequence * a.pages.ld_table, (uint32_t)position);
    auto target = [&](uint32_t h) { return h < a.heads ? q_out + (size_t)h * a.dim * es : at < 0 ? nullptr : a.k_cache + at + (h - a.heads) * a.pages.stride_head; };

    /* the angle in full turns, its whole ones taken off before it is narrowed: far positions lose nothing */
    for (uint32_t j = threadIdx.x; j < a.half; j += blockDim.x) {
        const double turns = (double)position * (double)a.inv_freq[j] * 0.15915494309189533577;
        sincospif((float)(2.0 * (turns - rint(turns))), &s_sin[j], &s_cos[j]);
    }
    __syncthreads();
    if constexpr (V > 1) asm volatile("cp.async.wait_group 0;" ::: "memory");
    /* values: copied */
    if (at >= 0) {
        char *const to = a.v_cache + at + vi * V * es;
        for (uint32_t h = vfirst; h < values; h += vstep) {
            Piece<DT, V> w;
            if (V > 1 && h == vfirst) w.load_shared(slot(2 * B));
            else w.load(v + (size_t)h * a.dim * es);
            w.store(to + h * a.pages.stride_head);
        }
    }
    uint32_t b = 0;
    for (uint32_t h = first; h < heads; h += step, ++b) {
        char *const to = target(h);
        if (!to) continue;
        Piece<DT, V> p, r;
        if (V > 1 && b < B) {
            p.load_shared(slot(2 * b));
            if (two) r.load_shared(slot(2 * b + 1));
        } else {
            p.load(source(h) + x * es);
            if (two) r.load(source(h) + y * es);
        }
        if (turn) {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float c = s_cos[i * n + e], s = s_sin[i * n + e];
                const float u = p.get(kOne ? 2 * e : e), w = kOne ? p.get(2 * e + 1) : r.get(e);
                const float first_of = u * c - w * s, second_of = u * s + w * c;
                if (kOne) { p.set(2 * e, first_of); p.set(2 * e + 1, second_of); }
                else { p.set(e, first_of); r.set(e, second_of); }
            }
        }
        p.store(to + x * es);
        if (two) r.store(to + y * es);
    }
}

}  /* namespace sifar */

using namespace sifar;

extern "C" int sifar_cache_append(const sifar_cache_append_args *g, void *stream)
{
    static const char *fn = "sifar_cache_append";
    if (!g) { set_error("%s: no argument block", fn); return SIFAR_ERR_INVALID; }
    CacheShape c;
    if (int rc = check_cache(fn, c, g->dtype, g->kv_heads, g->head_dim, g->pages, g->page_size, g->max_pages, g->sequences, g->ld_page_table,
                             g->stride_page, g->stride_token, g->stride_head)) return rc;
    if (g->heads < 0 || ((size_t)g->heads + (size_t)g->kv_heads) * (size_t)g->head_dim >= (1u << 20) || g->rotary_dim < 0 || g->rotary_dim > g->head_dim ||
        g->rotary_dim % 2 || g->tokens >= kMaxRows) {
        set_error("%s: need heads >= 0, (heads + kv_heads) * head_dim below 2^20, an even rotary_dim of 0 .. head_dim and tokens below 2^31", fn);
        return SIFAR_ERR_INVALID;
    }
    if (g->tokens == 0) return SIFAR_OK;
    if (!g->k || !g->v || !g->k_cache || !g->v_cache || !g->position || (g->heads && (!g->q || !g->q_out)) || (!g->heads && (g->q || g->q_out)) ||
        (!g->page_table && c.max_pages && c.sequences) || (!g->inv_freq && g->rotary_dim)) {
        set_error("%s: k, v, the caches, page_table and position are needed, inv_freq to turn, q and q_out where there are heads", fn);
        return SIFAR_ERR_INVALID;
    }
    const size_t es = c.es, T = g->tokens, nq = (size_t)g->heads * c.dim, nk = (size_t)g->kv_heads * c.dim;
    const auto ld = [](size_t given, size_t cols) { return given ? given : cols; };
    const RowArray q{"q", g->q, T, nq, ld(g->ld_q, nq), es, false}, k{"k", g->k, T, nk, ld(g->ld_k, nk), es, false};
    const RowArray v{"v", g->v, T, nk, ld(g->ld_v, nk), es, false}, q_out{"q_out", g->q_out, T, nq, ld(g->ld_q_out, nq), es, true};
    const size_t entries = c.sequences ? (c.sequences - 1) * c.ld_table + c.max_pages : 0;
    const RowArray table{"page_table", g->page_table, 1, entries, entries, sizeof(int), false};
    const RowArray sequence{"sequence", g->sequence, 1, T, T, sizeof(int), false}, position{"position", g->position, 1, T, T, sizeof(int), false};
    const size_t half = (size_t)g->rotary_dim / 2;
    const RowArray freq{"inv_freq", g->inv_freq, 1, half, half, sizeof(float), false};
    const bool in_place = g->q && g->q == g->q_out && (q.ld == q_out.ld || T == 1);
    RowArray all[8] = {k, v, q_out, table, sequence, position, freq, q};
    if (int rc = check_arrays(fn, all, in_place ? 7 : 8)) return rc;
    if (int rc = check_array(fn, q)) return rc;
    const size_t extent = cache_extent(c);
    const RowArray kc{"k_cache", g->k_cache, 1, 1, 1, es, true}, vc{"v_cache", g->v_cache, 1, 1, 1, es, true};
    if (int rc = check_array(fn, kc)) return rc;
    if (int rc = check_array(fn, vc)) return rc;
    for (const RowArray &x : all)
        if (touches(x, g->k_cache, extent) || touches(x, g->v_cache, extent)) { set_error("%s: the cache overlaps %s", fn, x.name); return SIFAR_ERR_INVALID; }
    const long long apart = (long long)((intptr_t)g->v_cache - (intptr_t)g->k_cache);
    if (c.pages && (apart % (long long)es || rows_meet(c, apart / (long long)es, 0))) { set_error("%s: v_cache overlaps k_cache", fn); return SIFAR_ERR_INVALID; }

    AppendArgs a;
    a.q = (const char *)g->q; a.k = (const char *)g->k; a.v = (const char *)g->v;
    a.q_out = (char *)g->q_out; a.k_cache = (char *)g->k_cache; a.v_cache = (char *)g->v_cache;
    a.sequence = g->sequence; a.position = g->position; a.inv_freq = g->inv_freq;
    a.pages = device_pages(c, g->page_table);
    a.ld_q = q.ld * es; a.ld_k = k.ld * es; a.ld_v = v.ld * es; a.ld_q_out = q_out.ld * es;
    a.sequences = (uint32_t)c.sequences;
    a.heads = (uint32_t)g->heads; a.kv_heads = (uint32_t)g->kv_heads; a.dim = (uint32_t)c.dim; a.half = (uint32_t)half;
    /* 16-byte pieces where every head's row and both halves of what turns are whole ones */
    const size_t per = 16 / es;
    const bool inter = g->interleaved != 0;
    const bool vec = rows_aligned16(q) && rows_aligned16(k) && rows_aligned16(v) && rows_aligned16(q_out) && cache_aligned16(c, g->k_cache, g->v_cache) &&
                     c.dim % per == 0 && (inter ? 2 * half : half) % per == 0;
    const size_t V = vec ? per : 1;
    a.turned = (uint32_t)((inter && vec ? 2 * half : half) / V + (c.dim - 2 * half) / V);
    a.copied = (uint32_t)(c.dim / V);
    /* up to 256 threads, 512 for few tokens: about two items of each */
    const size_t items = ((size_t)a.heads + a.kv_heads) * a.turned, most = T < 2 * kSms ? 512 : 256;
    size_t threads = 64;
    while (threads < a.turned || threads < a.copied || (threads < most && threads * 2 < items)) threads *= 2;
    const size_t shared = vec ? threads * 5 * 16 : 0;                /* two items of a key or query head, one of a value's */
    const dim3 grid((unsigned)T), block((unsigned)threads);
    const cudaStream_t st = (cudaStream_t)stream;
    cudaError_t err;
    if (g->dtype == SIFAR_BF16)
        err = !vec ? (inter ? launch_op(k_append<SIFAR_BF16, 1, true>, grid, block, 1, shared, st, a) : launch_op(k_append<SIFAR_BF16, 1, false>, grid, block, 1, shared, st, a))
                   : (inter ? launch_op(k_append<SIFAR_BF16, 8, true>, grid, block, 1, shared, st, a) : launch_op(k_append<SIFAR_BF16, 8, false>, grid, block, 1, shared, st, a));
    else
        err = !vec ? (inter ? launch_op(k_append<SIFAR_F32, 1, true>, grid, block, 1, shared, st, a) : launch_op(k_append<SIFAR_F32, 1, false>, grid, block, 1, shared, st, a))
                   : (inter ? launch_op(k_append<SIFAR_F32, 4, true>, grid, block, 1, shared, st, a) : launch_op(k_append<SIFAR_F32, 4, false>, grid, block, 1, shared, st, a));
    SIFAR_CUDA(err);
    return SIFAR_OK;
}
