/*
 * The paged cache as its two operators see it: addresses on the device, checks of the layout on the host.
 */
#ifndef SIFAR_CACHE_CUH
#define SIFAR_CACHE_CUH

#include "sifar_ops.cuh"

namespace sifar {

/* Strides in bytes. */
struct Pages {
    const int *table;
    unsigned long long ld_table;         /* entries between two sequences */
    unsigned long long stride_page, stride_token, stride_head;
    uint32_t pages, page_size, max_pages;
    uint32_t magic, shift;               /* n / page_size = n * magic >> 32 >> shift for n < 2^31; page_size 1: magic 0 */
};

/* Number of the page that holds token n, and n's place in it. */
__device__ __forceinline__ uint32_t page_of(const Pages &p, uint32_t n, uint32_t &in)
{
    const uint32_t at = p.magic ? __umulhi(n, p.magic) >> p.shift : n;
    in = n - at * p.page_size;
    return at;
}
/* Bytes from the start of the cache to place `in` of a page (its first head), or -1 where there is no such page. */
__device__ __forceinline__ long long place_offset(const Pages &p, int page, uint32_t in)
{
    if ((uint32_t)page >= p.pages) return -1;                 /* negative ones too */
    return (long long)((unsigned long long)page * p.stride_page + (unsigned long long)in * p.stride_token);
}

/* Bytes from the start of the cache to token n of a sequence (its first head), or -1 where the page is not there.  (A plain load: the
   kernel in front may have written the table while this one was started, so the table is not constant for this kernel's life.) */
__device__ __forceinline__ long long token_offset(const Pages &p, const int *row, uint32_t n)
{
    uint32_t in;
    const uint32_t at = page_of(p, n, in);
    return at < p.max_pages ? place_offset(p, row[at], in) : -1;
}

/* ------------------------------------------------------------------------ */
/* host                                                                      */
/* ------------------------------------------------------------------------ */
struct CacheShape {
    size_t pages, page_size, max_pages, sequences, ld_table;
    size_t stride[3], count[3];          /* outermost first; elements */
    size_t stride_page, stride_token, stride_head;
    size_t dim, es;
};

/* Whether rows at multiples of the strides, `shift` elements apart, share an element: shift = sum of a_i stride_i + rest
   with |a_i| < count_i and |rest| < dim.  Each stride holds what lies within it, so only two values of a_i can do. */
inline bool rows_meet(const CacheShape &c, long long shift, int level)
{
    if (level == 3) return shift > -(long long)c.dim && shift < (long long)c.dim;
    const long long s = (long long)c.stride[level], n = (long long)c.count[level];
    long long a = shift / s;
    if (shift % s < 0) --a;
    for (long long i = a; i <= a + 1; ++i)
        if (i > -n && i < n && rows_meet(c, shift - i * s, level + 1)) return true;
    return false;
}

/* Bytes from the first element to behind the last. */
inline size_t cache_extent(const CacheShape &c)
{
    if (c.pages == 0) return 0;
    size_t n = c.dim;
    for (int i = 0; i < 3; ++i) n += (c.count[i] - 1) * c.stride[i];
    return n * c.es;
}

inline int check_cache(const char *fn, CacheShape &c, int dtype, int kv_heads, int head_dim, size_t pages, size_t page_size, size_t max_pages,
                       size_t sequences, size_t ld_table, size_t stride_page, size_t stride_token, size_t stride_head)
{
    constexpr size_t kInts = (size_t)1 << 31, kFar = (size_t)1 << 45;
    if ((dtype != SIFAR_BF16 && dtype != SIFAR_F32) || kv_heads < 1 || kv_heads > 65535 || head_dim < 1 || head_dim > SIFAR_CACHE_MAX_HEAD_DIM) {
        set_error("%s: need dtype in {0,1}, 1 <= kv_heads <= 65535 and 1 <= head_dim <= %d", fn, (int)SIFAR_CACHE_MAX_HEAD_DIM);
        return SIFAR_ERR_INVALID;
    }
    if (page_size < 1 || page_size >= kInts || pages >= kInts || max_pages >= kInts || max_pages * page_size >= kInts || sequences >= kInts ||
        (ld_table && ld_table < max_pages) || ld_table >= kInts) {
        set_error("%s: need page_size >= 1, page counts, sequences and max_pages * page_size below 2^31 and ld_page_table of at least max_pages", fn);
        return SIFAR_ERR_INVALID;
    }
    c.pages = pages; c.page_size = page_size; c.max_pages = max_pages; c.sequences = sequences;
    c.ld_table = ld_table ? ld_table : max_pages;
    c.dim = (size_t)head_dim; c.es = elem_size(dtype);
    if (!stride_page && !stride_token && !stride_head) {
        stride_head = c.dim;
        stride_token = stride_head * (size_t)kv_heads;
        stride_page = stride_token * page_size;
    }
    if (stride_page >= kFar || stride_token >= kFar || stride_head >= kFar) { set_error("%s: a cache stride is too large", fn); return SIFAR_ERR_INVALID; }
    c.stride_page = stride_page; c.stride_token = stride_token; c.stride_head = stride_head;
    /* one of a kind: its stride is not used, and takes the place of the extent inside */
    const size_t hs = kv_heads == 1 ? 0 : stride_head, ts = page_size == 1 ? 0 : stride_token;
    const bool heads_inside = hs <= ts || ts == 0;
    size_t inner = c.dim;
    bool fits = true;
    for (int i = 2; i >= 1; --i) {
        const bool head = heads_inside == (i == 2);
        const size_t n = head ? (size_t)kv_heads : page_size;
        const size_t s = n == 1 ? inner : head ? stride_head : stride_token;
        fits = fits && s >= inner;
        c.count[i] = n; c.stride[i] = s;
        inner += (n - 1) * s;
    }
    c.count[0] = pages ? pages : 1;
    c.stride[0] = pages <= 1 ? inner : stride_page;
    if (!fits || c.stride[0] < inner || inner >= kFar) {
        set_error("%s: rows of the cache overlap (stride_page %zu, stride_token %zu, stride_head %zu)", fn, stride_page, stride_token, stride_head);
        return SIFAR_ERR_INVALID;
    }
    return SIFAR_OK;
}

inline Pages device_pages(const CacheShape &c, const int *table)
{
    Pages p;
    p.table = table; p.ld_table = c.ld_table;
    p.stride_page = c.stride_page * c.es; p.stride_token = c.stride_token * c.es; p.stride_head = c.stride_head * c.es;
    p.pages = (uint32_t)c.pages; p.page_size = (uint32_t)c.page_size; p.max_pages = (uint32_t)c.max_pages;
    /* magic = 2^(31 + l) / page_size rounded up, 2^l the next power of two: n * magic / 2^(31 + l) is less than 1 / page_size above
       n / page_size */
    uint32_t l = 0;
    while (((uint64_t)1 << l) < c.page_size) ++l;
    p.magic = l ? (uint32_t)((((uint64_t)1 << (31 + l)) + c.page_size - 1) / c.page_size) : 0u;
    p.shift = l ? l - 1 : 0u;
    return p;
}

/* Whether all rows of the cache start on 16-byte boundaries. */
inline bool cache_aligned16(const CacheShape &c, const void *k, const void *v)
{
    bool ok = (((uintptr_t)k | (uintptr_t)v) & 15u) == 0;
    for (int i = 0; i < 3; ++i) ok = ok && (c.count[i] == 1 || c.stride[i] * c.es % 16 == 0);
    return ok;
}

/* Whether an array shares bytes with [p, p + n): the cache is looked at as one piece. */
inline bool touches(const RowArray &a, const void *p, size_t n)
{
    if (!a.p || !a.rows || !a.cols || !n) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)p;
    return x < y + n && y < x + ((a.rows - 1) * a.ld + a.cols) * a.es;
}

}  /* namespace sifar */
#endif
