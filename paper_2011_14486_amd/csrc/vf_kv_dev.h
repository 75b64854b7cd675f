// Device pieces that the attention operators share: a cache's pages and a call's sequences.
#pragma once

#include "vf_ops_dev.h"

namespace vfkv {

using namespace vfo;

template <int FMT> struct kv_elem;  // an element of a row as it lies in memory
template <> struct kv_elem<VF_FP32> { typedef float type; };
template <> struct kv_elem<VF_BF16> { typedef uint16_t type; };
template <> struct kv_elem<VF_E4M3> { typedef uint8_t type; };

struct Cache {
  void *k, *v;
  uint8_t *ks, *vs;
  int heads, dim, width, kb, shift, pages;  // width: elements of a row; kb: scales of one; a page has 1 << shift tokens
};
struct Seqs {
  const int32_t *offsets, *lengths, *table;
  int64_t ld_table, tokens;
  int n, max_pages, each;  // each: rows of every sequence without offsets
};
struct Span {
  int64_t first;  // its first row
  int rows, length;
};

inline Cache cache_of(const vf_kv *kv) {
  Cache c;
  c.k = kv->k_dev; c.v = kv->v_dev; c.ks = kv->k_scales_dev; c.vs = kv->v_scales_dev;
  c.heads = kv->kv_heads; c.dim = kv->head_dim; c.pages = kv->pages;
  c.kb = (kv->head_dim + 31) / 32;
  c.width = kv->format == VF_E4M3 ? 32 * c.kb : (kv->head_dim + 7) / 8 * 8;
  c.shift = __builtin_ctz((unsigned)kv->page);
  return c;
}
inline Seqs seqs_of(const vf_kv_seqs *s) {
  Seqs q;
  q.offsets = s->offsets_dev; q.lengths = s->lengths_dev; q.table = s->table_dev; q.ld_table = s->ld_table; q.tokens = s->tokens;
  q.n = s->n_seq; q.max_pages = s->max_pages;
  q.each = s->n_seq > 0 && !s->offsets_dev ? (int)(s->tokens / s->n_seq) : 0;
  return q;
}
// r / by for r below 2^31: with 2^(s - 1) < by <= 2^s and magic = 2^(31 + s) / by rounded up, the product is off by less than
// r by <= 2^(31 + s) at the most, in units of 1 / by below the next quotient.
struct Divisor {
  uint32_t magic;
  int shift, by;
};
inline Divisor divisor_of(int by) {
  int s = 0;
  while (((int64_t)1 << s) < by) ++s;
  Divisor d;
  d.by = by;
  d.shift = 31 + s;
  d.magic = (uint32_t)((((uint64_t)1 << d.shift) + (uint64_t)by - 1) / (uint64_t)by);
  return d;
}
__device__ __forceinline__ int over(const Divisor &d, int r) { return (int)((uint64_t)(uint32_t)r * d.magic >> d.shift); }

// The most rows of a sequence, as the caller says where lengths differ.
inline int64_t longest_of(const vf_kv_seqs *s) {
  if (!s->offsets_dev) return s->n_seq > 0 ? s->tokens / s->n_seq : 0;
  return s->longest < s->tokens ? s->longest : s->tokens;
}

// Numbers that no kernel here writes, as constant memory: from an address that is the same in all lanes they come by a scalar load, which is waited for where
// it is used.  (A vector load of such a number would be waited for at once, and with it all loads that are on their way.)
__device__ __forceinline__ int fixed_at(const int32_t *p, int64_t i) {
  return ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)p)[i];
}

__device__ __forceinline__ Span span_of(const Seqs &q, int shift, int s) {
  Span p;
  p.first = (int64_t)s * q.each;
  p.rows = q.each;
  if (q.offsets) {
    const int b = fixed_at(q.offsets, s), e = fixed_at(q.offsets, (int64_t)s + 1);
    const bool fine = b >= 0 && e >= b && e <= q.tokens;
    p.first = fine ? b : 0;
    p.rows = fine ? e - b : 0;
  }
  const int most = q.max_pages << shift, n = fixed_at(q.lengths, s);
  p.length = n < 0 ? 0 : n > most ? most : n;
  return p;
}
// The entry of a sequence's table for position t >= 0; -1 behind the table's end.
__device__ __forceinline__ int entry_of(const Seqs &q, int shift, int s, int t) {
  const int at = t >> shift;
  return at < q.max_pages ? fixed_at(q.table, (int64_t)s * q.ld_table + at) : -1;
}
// Number of position t's row in a page of a head, over all pages and heads.
__device__ __forceinline__ int64_t row_of(const Cache &c, int page, int head, int t) {
  return (((int64_t)page * c.heads + head) << c.shift) + (t & ((1 << c.shift) - 1));
}

}  // namespace vfkv
