// Tensors of rows x heads x head_dim elements as the entry points take them.
#pragma once

#include "gbt_internal.h"

struct AttnView {   // rows x heads x head_dim elements; strides in elements, the head's elements side by side
    char *data;
    int64_t row, head;
};

namespace {

inline bool view_ok(const gbt_heads *h) {
    return h && ((uintptr_t)h->data & 15u) == 0 && h->row_stride >= 0 && h->head_stride >= 0 && h->row_stride % 8 == 0 && h->head_stride % 8 == 0 &&
           h->row_stride < ((int64_t)1 << 24) && h->head_stride < ((int64_t)1 << 40);
}
// No two of its heads' rows share elements: what is written to.
inline bool apart(const gbt_heads &h, int64_t rows, int64_t heads, int64_t dim) {
    int64_t near = h.row_stride, n_near = rows, far = h.head_stride, n_far = heads;
    if (n_far <= 1 || (n_near > 1 && near > far)) {
        std::swap(near, far);
        std::swap(n_near, n_far);
    }
    if (n_near <= 1) return n_far <= 1 || far >= dim;
    return near >= dim && (n_far <= 1 || (far - dim) / near >= n_near - 1);
}
inline AttnView view(const gbt_heads *h) { return AttnView{(char *)h->data, h->row_stride, h->head_stride}; }

}  // namespace

#define GBT_VIEW(ctx, h, rows)                                                                                                        \
    GBT_REQUIRE(ctx, view_ok(h), GBT_EINVAL, #h ": NULL, not 16-byte aligned, or strides that are negative, no multiples of 8 or (rows) 2^24 and more");    \
    GBT_REQUIRE(ctx, (h)->data || (rows) == 0, GBT_EINVAL, #h ": data is NULL")
#define GBT_VIEW_OUT(ctx, h, rows, heads)                                                                                             \
    GBT_VIEW(ctx, h, rows);                                                                                                           \
    GBT_REQUIRE(ctx, apart(*(h), rows, heads, p.head_dim), GBT_EINVAL, #h ": rows or heads overlap")
