// Checks of the arguments that every call on the paged cache of 8-bit floating point takes.
#ifndef KVQ_PAGED8_HOST_H
#define KVQ_PAGED8_HOST_H

#include <algorithm>
#include <cstdint>
#include <cstdlib>

#include "../../include/kvq.h"
#include "kvq_paged8.h"

inline bool kvq_p8_aligned(const void* p, uintptr_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline bool kvq_p8_args(const kvq_paged8_t* c, const kvq_paged8_batch_t* b, KvqP8& P) {
    if (!c || !b) return false;
    int shift = 0;
    for (int s = 5; s <= 8; ++s)
        if (c->page_tokens == 1 << s) shift = s;
    if (!shift || c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535) return false;
    if (b->n_seqs < 0 || b->n_seqs > KVQ_P8_MOST_SEQS || b->n_rows < 0 || b->n_rows > INT32_MAX / 64) return false;
    if (b->max_rows < 1 || b->table_pages < 1 || b->table_pages > (INT32_MAX - 4096) >> shift) return false;
    if (b->table_stride < (b->n_seqs > 1 ? b->table_pages : 0) || b->table_stride >= (1ll << 40)) return false;
    if (!kvq_p8_aligned(c->codes_dev, 16) || !kvq_p8_aligned(c->words_dev, 8)) return false;
    if (b->n_seqs && (!kvq_p8_aligned(b->table_dev, 4) || !kvq_p8_aligned(b->lengths_dev, 4))) return false;
    if (reinterpret_cast<uintptr_t>(b->row_begin_dev) & 3u) return false;
    if (!b->row_begin_dev && b->n_rows < b->n_seqs) return false;
    P.codes = static_cast<uint8_t*>(c->codes_dev);
    P.words = c->words_dev;
    P.table = b->table_dev;
    P.lengths = b->lengths_dev;
    P.row_begin = b->row_begin_dev;
    P.table_stride = b->table_stride;
    P.n_pages = c->n_pages;
    P.n_kv = c->n_kv_heads;
    P.page_shift = shift;
    P.table_pages = b->table_pages;
    P.n_seqs = b->n_seqs;
    P.n_rows = b->n_rows;
    P.max_rows = b->row_begin_dev ? std::min(b->max_rows, std::max(1, b->n_rows)) : 1;
    return true;
}
// Rows of 128 values by 16-byte accesses; `align`: elements that 16 bytes hold.
inline bool kvq_p8_rows_ok(const kvq_paged8_rows_t* r, const kvq_paged8_batch_t* b, int align) {
    if (!r) return false;
    for (int64_t s : {r->row_stride, r->head_stride})
        if (s < 0 || s % align != 0 || s >= (1ll << 40)) return false;
    return b->n_rows == 0 || kvq_p8_aligned(r->data_dev, 16);
}
// Whether no two of the rows t * row + h * head, 128 long each, share an element (strides of 128 or more).
inline bool kvq_p8_rows_apart(const kvq_paged8_rows_t* r, const kvq_paged8_batch_t* b, int64_t heads) {
    const int64_t row = r->row_stride, head = r->head_stride, n = b->n_rows;
    if ((n > 1 && row < KVQ_D) || (heads > 1 && head < KVQ_D)) return false;
    if (n <= 1 || heads <= 1 || row >= (heads - 1) * head + KVQ_D || head >= (n - 1) * row + KVQ_D) return true;
    for (int64_t h = 1; h < heads; ++h)  // the rows that h heads on comes next to
        for (int64_t t = h * head / row, k = 0; k < 2; ++k, ++t)
            if (t < n && std::abs(h * head - t * row) < KVQ_D) return false;
    return true;
}

#endif
