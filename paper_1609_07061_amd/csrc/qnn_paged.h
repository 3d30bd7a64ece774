// Shared by the calls on heads and the paged cache (qnn_heads.hip, qnn_cache_attention.hip): where a token of a sequence lies, and what the host checks.
#pragma once
#include "qnn_rows.h"

namespace qnn {
namespace paged {

constexpr int kMostD = 256;
constexpr uint32_t kNoRow = 0xFFFFFFFFu;  // (rows of the cache are below it)

struct Pages {
    const int32_t *table;
    int64_t ld, width;
    uint32_t pages, heads, page, page_inverse;  // page_inverse: inverse_of(page)
};
// Where token `at` of a sequence is: the page's number, as the table has it (kNoRow beyond the table), and the place in it.  at >= 0
struct Place {
    uint32_t id, in_page;
};
__device__ __forceinline__ Place place_of(const Pages &p, int64_t sequence, uint32_t at) {
    Place x;
    const uint32_t number = quotient(at, p.page, p.page_inverse, x.in_page);
    x.id = (int64_t)number < p.width ? (uint32_t)p.table[sequence * p.ld + number] : kNoRow;
    return x;
}
// The row of the cache for a head, kNoRow without one.  (A step of its own: what asks for the number need not wait for it.)
__device__ __forceinline__ uint32_t row_of(const Pages &p, const Place &x, uint32_t head) {
    return x.id < p.pages ? (x.id * p.heads + head) * p.page + x.in_page : kNoRow;
}
inline Pages pages_of(const qnn_paged_cache &c) {
    return {c.table, c.ld_table, c.width, (uint32_t)c.pages, (uint32_t)c.heads, (uint32_t)c.page, inverse_of(c.page)};
}

inline int check_cache(const char *what, const qnn_paged_cache *c) {
    if (!c) return fail(QNN_ERR_NULL, "%s: NULL cache", what);
    if (c->pages < 1 || c->heads < 1 || c->page < 1 || c->sequences < 0 || c->width < 0 || c->ld_table < c->width)
        return fail(QNN_ERR_SHAPE, "%s: %lld pages of %lld tokens, %lld heads, %lld sequences, table %lld of %lld", what, (long long)c->pages, (long long)c->page,
                    (long long)c->heads, (long long)c->sequences, (long long)c->width, (long long)c->ld_table);
    if (c->D < 16 || c->D > kMostD || c->D % 16) return fail(QNN_ERR_UNSUPPORTED, "%s: heads of %lld values (a multiple of 16, at most 256)", what, (long long)c->D);
    if ((double)c->pages * (double)c->heads * (double)c->page >= 4294967296.0 || c->page > 0x3FFFFFFF || c->sequences > 0x3FFFFFFF)
        return fail(QNN_ERR_UNSUPPORTED, "%s: a cache of 2^32 rows or more", what);
    return QNN_OK;
}
inline int check_cache_pointers(const char *what, const qnn_paged_cache *c) {
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->starts || !c->lengths || (!c->table && c->width > 0)) return fail(QNN_ERR_NULL, "%s: NULL pointer in the cache", what);
    if (!rows::aligned_to(c->k, 16) || !rows::aligned_to(c->v, 16)) return fail(QNN_ERR_ALIGN, "%s: codes not aligned to 16 bytes", what);
    if (!rows::aligned_to(c->k_scale, 4) || !rows::aligned_to(c->v_scale, 4) || !rows::aligned_to(c->starts, 4) || !rows::aligned_to(c->lengths, 4) ||
        !rows::aligned_to(c->table, 4))
        return fail(QNN_ERR_ALIGN, "%s: pointer in the cache not aligned to its type", what);
    return QNN_OK;
}
// A matrix of heads: value d of head h of token t at t * ld + h * step + d.  Rows of heads must not overlap.
inline bool heads_fit(int64_t ld, int64_t step, int64_t heads, int64_t D, int64_t tokens) {
    if (heads < 1) return true;
    if ((heads > 1 && step < D) || step < 0 || ld < 0) return false;
    if (tokens <= 1) return true;
    // heads within a token's row, or tokens within a head's
    return ld >= (heads - 1) * step + D || (heads > 1 && ld >= D && step >= (tokens - 1) * ld + D);
}

}  // namespace paged
}  // namespace qnn
