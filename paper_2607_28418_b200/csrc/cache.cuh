// The 4-bit paged key/value cache as the kernels see it: addresses, the new rows of a sequence, levels.
#pragma once

#include "internal.h"

constexpr int WIDE_MAX_LEN = 0x7ffffff0;   // of a sequence: rounded up to whole blocks it stays an int

struct CacheView {
    uint8_t* pages;
    int n_pages, page_shift, n_kv_heads;   // page_size = 1 << page_shift
    int block_bytes;                       // 16 tokens of one head
};

struct SeqView {
    const int32_t* page_table;
    const int32_t* kv_lens;
    const int32_t* row_start;
    int n_seqs, max_pages, rows;
};

// One sequence after its checks: rows [row0, row0 + n_rows) are the positions [len - n_rows, len).
// n_rows = 0 where the row range is not usable; len = 0 where the length is not.
struct SeqInfo {
    int row0, n_rows, len;
    bool bad;
};

#ifdef __CUDACC__
__device__ __forceinline__ SeqInfo wide_seq_info(const SeqView& q, int s, int page_shift) {
    SeqInfo i;
    int a = s, b = s + 1;
    if (q.row_start) {
        a = q.row_start[s];
        b = q.row_start[s + 1];
    }
    const bool rows_ok = a >= 0 && b >= a && b <= q.rows;
    const int len = q.kv_lens[s];
    const bool len_ok = len >= 0 && len <= WIDE_MAX_LEN && static_cast<long long>(len) <= (static_cast<long long>(q.max_pages) << page_shift) &&
                        (!rows_ok || len >= b - a);
    i.row0 = a;
    i.n_rows = rows_ok ? b - a : 0;
    i.len = len_ok ? len : 0;
    i.bad = !rows_ok || !len_ok;
    return i;
}

// Address of the 16-token block that holds position p of sequence s for one head; nullptr where the page
// table names no page.  All products in 64 bits: a cache is far larger than 2^32 bytes.
__device__ __forceinline__ uint8_t* wide_cache_block(const CacheView& c, const SeqView& q, int s, int p, int head) {
    const int page = q.page_table[static_cast<size_t>(s) * q.max_pages + (p >> c.page_shift)];
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(c.n_pages)) return nullptr;
    const int sub = (p & ((1 << c.page_shift) - 1)) >> 4;
    const size_t block = ((static_cast<size_t>(page) * c.n_kv_heads + head) << (c.page_shift - 4)) + sub;
    return c.pages + block * c.block_bytes;
}

// the two halves of a parameter word
__device__ __forceinline__ float wide_cache_scale(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float wide_cache_min(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
#endif

inline CacheView wide_cache_view(const wide_cache* c) {
    CacheView v;
    v.pages = static_cast<uint8_t*>(c->pages);
    v.n_pages = c->n_pages;
    v.page_shift = 31 - __builtin_clz(static_cast<unsigned>(c->page_size));
    v.n_kv_heads = c->n_kv_heads;
    v.block_bytes = 16 * c->head_dim + 128 * (c->head_dim / c->quant_group);
    return v;
}
inline SeqView wide_seq_view(const wide_seqs* s, int rows) {
    return SeqView{s->page_table, s->kv_lens, s->row_start, s->n_seqs, s->max_pages, rows};
}
