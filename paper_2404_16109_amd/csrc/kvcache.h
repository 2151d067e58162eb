// The cache of 8-bit keys and values as its kernels see it.
#pragma once
#include "serve_dev.h"

namespace zkmi {

// One sequence of a call, or why it is skipped.
struct SeqView {
    int32_t row0, rows, len;  // its rows in the call's tensors, its length with them
    bool ok;
};

__device__ __forceinline__ SeqView seq_view(const kv_seqs& s, uint32_t b, uint32_t page_log) {
    SeqView v;
    v.row0 = s.cu[b];
    const int32_t end = s.cu[b + 1];
    v.rows = end - v.row0;
    v.len = s.lens[b];
    v.ok = v.row0 >= 0 && end >= v.row0 && (uint32_t)end <= s.rows && (uint32_t)v.rows <= s.max_new && v.len >= 0 &&
           ((uint64_t)v.len + (1u << page_log) - 1) >> page_log <= s.table_pages;
    return v;
}

__device__ __forceinline__ void report(const kv_seqs& s, uint32_t what) {
    if (s.fault) atomicOr(s.fault, what);
}

inline bool page_size_ok(uint32_t t) { return is_pow2(t) && t >= 16 && t <= 256; }
inline bool cache_ok(const kvcache_i8* c) {
    return c && c->k && c->v && c->k_exp && c->v_exp && aligned(c->k, 16) && aligned(c->v, 16) && c->pages >= 1 && c->pages < 0x80000000u &&
           c->kv_heads >= 1 && c->kv_heads <= 16384 && page_size_ok(c->page_tokens) && c->head_dim >= 16 && c->head_dim <= 256 &&
           c->head_dim % 16 == 0;
}
inline bool seqs_ok(const kv_seqs* s) {
    return s && s->cu && s->lens && s->table && aligned(s->cu, 4) && aligned(s->lens, 4) && aligned(s->table, 4) && s->seqs <= 65535 &&
           s->rows < 0x80000000u && s->max_new >= 1 && (!s->fault || aligned(s->fault, 4)) &&
           s->table_pages >= 1 && (s->seqs <= 1 || s->table_stride >= s->table_pages);
}

}  // namespace zkmi
