// The paged cache as kernels see it: sequences, pages, visibility.
#pragma once
#include "internal.h"

namespace pcm {

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31: with s = ceil(log2 d) and m = ceil(2^(31+s) / d) < 2^32 the error of
// n m / 2^(31+s) is below n / (2^31 d) < 1 / d, so the floor is right.
struct FastDiv { unsigned d, m; int shift; };
static inline FastDiv make_fastdiv(int d) {
  FastDiv f;
  int s = 0;
  while ((1ll << s) < d) ++s;
  f.d = (unsigned)d; f.shift = 31 + s;
  f.m = (unsigned)(((1ull << f.shift) + (unsigned)d - 1) / (unsigned)d);
  return f;
}
__device__ __forceinline__ int fast_div(int n, const FastDiv& f) { return (int)(((unsigned long long)(unsigned)n * f.m) >> f.shift); }

struct KvView {
  const void* k; const void* v;
  long long ld_page, ld_slot, ld_head;
  int n_pages, page_size, n_kv;
  FastDiv div_page;
  const int* table; long long ld_table;
  const int* seq_len;
  const int* q_off;
  int n_seq, n_rows;
  int max_len;                                 // tokens that a row of the table can hold
  unsigned* status;                            // pages and lengths that do not fit; may be null
  unsigned* waits;                             // expired waits: the call's own word, or the device's (kernels that wait)
};

__device__ __forceinline__ void kv_report(const KvView& c, unsigned bit) {
  if (c.status) atomicOr(c.status, bit);
}

__device__ __forceinline__ void kv_report_expired(const KvView& c) { atomicOr(c.waits, STATUS_TIMEOUT); }

struct SeqSpan { int row0, fresh, len; };      // first row and number of new tokens, tokens in all

// A sequence's rows and length, clipped to what the call's sizes allow.
__device__ __forceinline__ SeqSpan seq_span(const KvView& c, int s, bool report) {
  SeqSpan sp;
  int a = s, b = s + 1, len = c.seq_len[s];
  if (c.q_off) { a = c.q_off[s]; b = c.q_off[s + 1]; }
  bool bad = false;
  if (a < 0 || b < a || b > c.n_rows) { a = b = 0; bad = true; }
  if (len < 0 || len > c.max_len) { len = len < 0 ? 0 : c.max_len; bad = true; }
  if (bad && report) kv_report(c, STATUS_BAD_LENGTH);
  sp.row0 = a; sp.fresh = b - a; sp.len = len;
  return sp;
}

// Whether rows of heads that are written may share elements: neither do a row's heads end before the next row, nor a head's
// rows before the next head.
static inline bool rows_overlap(int64_t n, int64_t heads, int64_t dim, int64_t ld, int64_t ld_head) {
  if (n <= 1 || heads <= 1) return (n > 1 && ld < dim) || (heads > 1 && ld_head < dim);
  return ld < dim || ld_head < dim || (ld < (heads - 1) * ld_head + dim && ld_head < (n - 1) * ld + dim);
}

// Checks of the two structs that every call makes before it reads from them.
int kv_check(const grpo_kv_cache* cache, const grpo_kv_batch* batch, int32_t n_rows);
KvView kv_view(const grpo_kv_cache* cache, const grpo_kv_batch* batch, int32_t n_rows, uint32_t* status);

}  // namespace pcm
