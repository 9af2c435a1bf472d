// Rotary positions: of given rows (grpo_rotary, and its gradient as the opposite rotation), and of new tokens on their way
// into a paged cache (grpo_rotary_cache).
//
// A pair (a, b) of a head's elements at position t turns by the angle 2 pi t f: (a cos - b sin, b cos + a sin).  The whole
// turns of t f carry no information and would cost fp32 all of its digits at far positions, so t f is formed and reduced to
// [-1/2, 1/2] in 64 bits (error below 2^-22 turns at t = 2^31) and only the rest goes through sincospif.  All heads of a row share its
// angles: a block forms the sines and cosines of its rows once in shared memory, then streams the rows through them, each
// element read and written once: bound by HBM (119808 rows of 16 heads of 64 in bf16: 80 us, 6.1 TB/s, in fp32 150 us; 98304 new tokens of
// 16/8 heads into a cache: 130 us, 6.2 TB/s, in fp32 246 us; heads whose turning halves are no multiple of 16 bytes go by the element:
// 119808 x 16 x 96 in bf16 with 24 turning 721 us, 154 with 48; a step of 64 tokens: 6 us, which are dependent reads of offsets, lengths and table).
#include <cmath>

#include "paged.cuh"

namespace pcm {

constexpr int RT_THREADS = 256;
constexpr int RT_ANGLES = 2048;                // angles of a block's rows: 16 KB
constexpr int RT_ROWS = 16;                    // rows per block at most

struct RotaryStream {                          // n_heads heads of every row: source and destination
  const void* src; long long ld, ld_head;
  void* dst; long long ld_dst, ld_dst_head;
  int n_heads;
};
struct RotaryParams {
  RotaryStream q, k, v;                        // k and v go to the cache; plain rows are q alone
  int n, half, dim;
  const double* turns;
  float amplitude;
  int inverse;
  const int* pos;
  int rows;                                    // rows per block
  int turn_units, units;                       // units of a head that turn, and all of a head's
  int copy_units;                              // units of a head of v
  int row_units;                               // units of a row
  FastDiv div_row, div_head, div_copy;
  int to_cache;
  int q_in_place;                              // q's elements that do not turn are where they belong
  KvView cache;
};

template <typename T> struct RtVec { static constexpr int N = 16 / sizeof(T); };
__device__ __forceinline__ float rt_load(float x) { return x; }
__device__ __forceinline__ float rt_load(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void rt_store(float* p, float x) { *p = x; }
__device__ __forceinline__ void rt_store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// The sequence of a row (ascending offsets), or -1.
__device__ static int sequence_of(const KvView& c, int row) {
  if (!c.q_off) return row < c.n_seq ? row : -1;
  const int even = (int)((long long)row * c.n_seq / c.n_rows);     // right where all sequences bring as many rows
  if (c.q_off[even] <= row && row < c.q_off[even + 1]) return even;
  int lo = 0, hi = c.n_seq;                    // first s with q_off[s + 1] > row
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (c.q_off[mid + 1] > row) hi = mid; else lo = mid + 1;
  }
  return lo < c.n_seq && c.q_off[lo] <= row ? lo : -1;
}

// A unit is what one thread handles at a time: with VEC, 16 bytes (interleaved), or 16 bytes of either half; else one pair;
// of what does not turn, 16 bytes or one element.
template <typename T, bool VEC, bool INTER>
__global__ void __launch_bounds__(RT_THREADS, 8) rotary_kernel(const __grid_constant__ RotaryParams p) {
  constexpr int N = VEC ? RtVec<T>::N : 1;
  __shared__ float2 cs[RT_ANGLES];
  __shared__ int row_pos[RT_ROWS];
  __shared__ long long row_slot[RT_ROWS];      // first element of the row's slot in the cache; -1: none, -2: not a row of the call
  const int row_base = blockIdx.x * p.rows, n_here = min(p.rows, p.n - row_base);
  if ((int)threadIdx.x < n_here) {
    const int row = row_base + threadIdx.x;
    int t = 0;
    long long slot = -1;
    if (p.to_cache) {
      const int s = sequence_of(p.cache, row);
      if (s < 0) {
        slot = -2;
      } else {
        const SeqSpan sp = seq_span(p.cache, s, false);
        if (row >= sp.row0 && row < sp.row0 + sp.fresh) {
          // from the length as it was given: counted back from a clipped one new tokens would land on stored ones
          const int j = max(p.cache.seq_len[s], 0) - sp.fresh + (row - sp.row0);
          t = p.pos ? p.pos[row] : j;
          if (j >= 0 && j < p.cache.max_len) {
            const int at = fast_div(j, p.cache.div_page);
            const int page = p.cache.table[s * p.cache.ld_table + at];
            if (page < 0 || page >= p.cache.n_pages) kv_report(p.cache, STATUS_BAD_PAGE);
            else slot = page * p.cache.ld_page + (j - at * p.cache.page_size) * p.cache.ld_slot;
          }
        } else {
          slot = -2;
        }
      }
    } else {
      t = p.pos[row];
    }
    row_pos[threadIdx.x] = t;
    row_slot[threadIdx.x] = slot;
  }
  if (p.to_cache && p.cache.status)            // every sequence's sizes are looked at once, by the warps that have no row to place
    for (long long s = (long long)blockIdx.x * RT_THREADS + RT_THREADS - 1 - threadIdx.x; s < p.cache.n_seq; s += (long long)gridDim.x * RT_THREADS)
      seq_span(p.cache, (int)s, true);
  double turns = (int)threadIdx.x < n_here * p.half ? p.turns[threadIdx.x % p.half] : 0.0;      // on its way with the row's place
  __syncthreads();
  for (int i = threadIdx.x; i < n_here * p.half; i += RT_THREADS) {
    const int r = i / p.half;
    if (i != (int)threadIdx.x) turns = p.turns[i - r * p.half];
    const double part = (double)row_pos[r] * turns;
    float s, c;
    sincospif(2.f * (float)(part - rint(part)), &s, &c);
    cs[i] = make_float2(c * p.amplitude, (p.inverse ? -s : s) * p.amplitude);
  }
  __syncthreads();
  const int qk_units = (p.q.n_heads + p.k.n_heads) * p.units;
  for (int i = threadIdx.x; i < n_here * p.row_units; i += RT_THREADS) {
    const int r = fast_div(i, p.div_row);
    int u = i - r * p.row_units;
    const long long slot = row_slot[r];
    if (slot == -2) continue;
    const long long row = row_base + r;
    const T* src;
    T* dst;
    bool copy;
    int e;                                     // first element
    if (u < qk_units) {
      int h = fast_div(u, p.div_head);
      u -= h * p.units;
      const bool is_q = h < p.q.n_heads;
      if (!is_q) h -= p.q.n_heads;
      const RotaryStream& st = is_q ? p.q : p.k;
      src = (const T*)st.src + row * st.ld + h * st.ld_head;
      if (!is_q && slot < 0) continue;
      dst = is_q ? (T*)st.dst + row * st.ld_dst + h * st.ld_dst_head : (T*)st.dst + slot + h * st.ld_dst_head;
      copy = u >= p.turn_units;
      e = copy ? 2 * p.half + (u - p.turn_units) * N : u * N * (INTER && !VEC ? 2 : 1);
      if (copy && is_q && p.q_in_place) continue;
    } else {
      u -= qk_units;
      if (slot < 0) continue;
      const int h = fast_div(u, p.div_copy);
      src = (const T*)p.v.src + row * p.v.ld + h * p.v.ld_head;
      dst = (T*)p.v.dst + slot + h * p.v.ld_dst_head;
      copy = true;
      e = (u - h * p.copy_units) * N;
    }
    if (copy) {
      if (VEC) *reinterpret_cast<uint4*>(dst + e) = *reinterpret_cast<const uint4*>(src + e);
      else dst[e] = src[e];
      continue;
    }
    const float2* turn = cs + r * p.half;
    if (VEC && INTER) {
      union { uint4 q; T t[RtVec<T>::N]; } a, o;
      a.q = *reinterpret_cast<const uint4*>(src + e);
#pragma unroll
      for (int k = 0; k < N; k += 2) {
        const float2 w = turn[(e + k) >> 1];
        const float x = rt_load(a.t[k]), y = rt_load(a.t[k + 1]);
        rt_store(&o.t[k], fmaf(x, w.x, -y * w.y));
        rt_store(&o.t[k + 1], fmaf(y, w.x, x * w.y));
      }
      *reinterpret_cast<uint4*>(dst + e) = o.q;
    } else if (VEC) {
      union { uint4 q; T t[RtVec<T>::N]; } a, b, oa, ob;
      a.q = *reinterpret_cast<const uint4*>(src + e);
      b.q = *reinterpret_cast<const uint4*>(src + e + p.half);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float2 w = turn[e + k];
        const float x = rt_load(a.t[k]), y = rt_load(b.t[k]);
        rt_store(&oa.t[k], fmaf(x, w.x, -y * w.y));
        rt_store(&ob.t[k], fmaf(y, w.x, x * w.y));
      }
      *reinterpret_cast<uint4*>(dst + e) = oa.q;
      *reinterpret_cast<uint4*>(dst + e + p.half) = ob.q;
    } else {
      const int far = INTER ? 1 : p.half;
      const float2 w = turn[INTER ? e >> 1 : e];
      const float x = rt_load(src[e]), y = rt_load(src[e + far]);
      rt_store(dst + e, fmaf(x, w.x, -y * w.y));
      rt_store(dst + e + far, fmaf(y, w.x, x * w.y));
    }
  }
}

template <typename T>
static int launch_rotary(RotaryParams p, bool inter, cudaStream_t s) {
  constexpr int N = RtVec<T>::N;
  // 16-byte accesses: every address that a unit may start at has to be a multiple of them (strides of one row or one head
  // lead nowhere)
  uintptr_t bits = 0;
  for (RotaryStream* st : {&p.q, &p.k, &p.v}) {
    if (p.n == 1) st->ld = st->ld_dst = 0;
    if (st->n_heads == 1) st->ld_head = st->ld_dst_head = 0;
    if (st->n_heads > 0)
      bits |= (uintptr_t)st->src | (uintptr_t)st->dst | (uintptr_t)((st->ld | st->ld_head | st->ld_dst | st->ld_dst_head) * sizeof(T));
  }
  const bool vec = !(bits & 15) && p.dim % N == 0 && (inter ? 2 * p.half : p.half) % N == 0;
  const int step = vec ? N : 1;
  p.turn_units = vec && inter ? 2 * p.half / N : p.half / step;
  p.copy_units = p.dim / step;
  p.units = p.turn_units + (p.dim - 2 * p.half) / step;
  const long long row_units = (long long)(p.q.n_heads + p.k.n_heads) * p.units + (long long)p.v.n_heads * p.copy_units;
  if (row_units * RT_ROWS > 0x7FFFFFFFll) return PCM_ERR_SHAPE;
  p.row_units = (int)row_units;
  p.div_row = make_fastdiv(p.row_units);
  p.div_head = make_fastdiv(p.units);
  p.div_copy = make_fastdiv(p.copy_units);
  // four units a thread, while that leaves four blocks for every SM and the angles fit
  p.rows = 1;
  while (p.rows < RT_ROWS && p.rows * row_units < 4 * RT_THREADS && p.n / (2 * p.rows) >= 4 * sm_count() &&
         2 * p.rows * p.half <= RT_ANGLES)
    p.rows *= 2;
  auto kernel = vec ? (inter ? rotary_kernel<T, true, true> : rotary_kernel<T, true, false>)
                    : (inter ? rotary_kernel<T, false, true> : rotary_kernel<T, false, false>);
  kernel<<<ceil_div(p.n, p.rows), RT_THREADS, 0, s>>>(p);
  PCM_LAUNCH_CHECK();
  return PCM_OK;
}

static bool dtype_known(int32_t dtype) { return dtype == GRPO_F32 || dtype == GRPO_BF16; }
static int elem_bytes(int32_t dtype) { return dtype == GRPO_BF16 ? 2 : 4; }

int kv_check(const grpo_kv_cache* c, const grpo_kv_batch* b, int32_t n_rows) {
  if (!c || !b || !dtype_known(c->dtype) || n_rows < 0 || b->n_seq < 0) return PCM_ERR_ARG;
  if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || b->max_pages < 1) return PCM_ERR_ARG;
  if (n_rows > PCM_MAX_VOCAB_CALL || b->n_seq > PCM_MAX_VOCAB_CALL || c->page_size % 8 || c->page_size > PCM_MAX_VOCAB_CALL) return PCM_ERR_SHAPE;
  if (b->n_seq == 0 || n_rows == 0) return PCM_OK;
  if (!c->k || !c->v || !b->page_table || !b->seq_len || b->ld_table < b->max_pages) return PCM_ERR_ARG;
  if (!b->q_off && n_rows != b->n_seq) return PCM_ERR_ARG;
  if (c->ld_page < 0 || c->ld_slot < 0 || c->ld_head < 0) return PCM_ERR_ARG;
  const int64_t per = 16 / elem_bytes(c->dtype);
  if ((((uintptr_t)c->k | (uintptr_t)c->v) & 15) || (c->n_pages > 1 && c->ld_page % per) || (c->ld_slot % per) ||
      (c->n_kv_heads > 1 && c->ld_head % per))
    return PCM_ERR_SHAPE;
  // neighbouring heads, slots and pages have room for a row of a head
  if ((c->n_kv_heads > 1 && c->ld_head < c->head_dim) || c->ld_slot < c->head_dim || (c->n_pages > 1 && c->ld_page < c->head_dim))
    return PCM_ERR_ARG;
  return PCM_OK;
}

KvView kv_view(const grpo_kv_cache* c, const grpo_kv_batch* b, int32_t n_rows, uint32_t* status) {
  KvView v;
  v.k = c->k; v.v = c->v;
  v.ld_page = c->n_pages > 1 ? c->ld_page : 0; v.ld_slot = c->ld_slot; v.ld_head = c->n_kv_heads > 1 ? c->ld_head : 0;
  v.n_pages = c->n_pages; v.page_size = c->page_size; v.n_kv = c->n_kv_heads;
  v.div_page = make_fastdiv(c->page_size);
  v.table = b->page_table; v.ld_table = b->ld_table;
  v.seq_len = b->seq_len; v.q_off = b->q_off;
  v.n_seq = b->n_seq; v.n_rows = n_rows;
  const long long hold = (long long)b->max_pages * c->page_size, most = PCM_MAX_VOCAB_CALL;
  v.max_len = (int)(hold < most ? hold : most);
  v.status = status;
  v.waits = status;
  return v;
}

}  // namespace pcm

using namespace pcm;

extern "C" int grpo_rotary_freqs(const grpo_rotary_cfg* cfg, double* turns, float* amplitude) {
  if (!cfg || !turns || !amplitude) return PCM_ERR_ARG;
  if (cfg->rot_dim < 2 || cfg->rot_dim % 2 || cfg->rot_dim > PCM_MAX_ROTARY_DIM) return PCM_ERR_SHAPE;
  if (!(cfg->base > 0.0) || !std::isfinite(cfg->base) || cfg->scaling < GRPO_ROTARY_PLAIN || cfg->scaling > GRPO_ROTARY_PARTS) return PCM_ERR_ARG;
  const bool squeezes = cfg->scaling != GRPO_ROTARY_PLAIN, parts = cfg->scaling == GRPO_ROTARY_PARTS;
  if (squeezes && (!(cfg->factor >= 1.0) || !std::isfinite(cfg->factor))) return PCM_ERR_ARG;
  if (cfg->scaling == GRPO_ROTARY_BASE && cfg->rot_dim < 4) return PCM_ERR_SHAPE;
  if (parts && (!(cfg->original_len > 0.0) || !std::isfinite(cfg->original_len) || !(cfg->low < cfg->high) || !std::isfinite(cfg->low) ||
                !std::isfinite(cfg->high)))
    return PCM_ERR_ARG;
  const double rot = cfg->rot_dim, two_pi = 6.283185307179586476925;
  const double base = cfg->scaling == GRPO_ROTARY_BASE ? cfg->base * std::pow(cfg->factor, rot / (rot - 2.0)) : cfg->base;
  for (int i = 0; i < cfg->rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot) / two_pi;
    if (cfg->scaling == GRPO_ROTARY_LINEAR) f /= cfg->factor;
    if (parts) {
      double keep = (cfg->original_len * f - cfg->low) / (cfg->high - cfg->low);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f *= keep + (1.0 - keep) / cfg->factor;
    }
    turns[i] = f;
  }
  *amplitude = parts ? (float)(0.1 * std::log(cfg->factor) + 1.0) : 1.f;
  return PCM_OK;
}

extern "C" int grpo_rotary(int32_t dtype, const void* x, int64_t ld_x, int64_t ld_x_head, int32_t n, int32_t n_heads, int32_t head_dim,
                           int32_t rot_dim, const double* turns, float amplitude, const int32_t* pos, uint32_t flags, void* out,
                           int64_t ld_out, int64_t ld_out_head, pcm_stream stream) {
  if (!dtype_known(dtype) || n < 0 || n_heads < 1 || head_dim < 1 || rot_dim < 0 || !std::isfinite(amplitude)) return PCM_ERR_ARG;
  if (flags & ~(GRPO_ROTARY_INTERLEAVED | GRPO_ROTARY_INVERSE)) return PCM_ERR_ARG;
  if (n > PCM_MAX_VOCAB_CALL || head_dim > PCM_MAX_ROTARY_DIM || rot_dim % 2 || rot_dim > head_dim || n_heads > (1 << 16)) return PCM_ERR_SHAPE;
  if (n == 0) return PCM_OK;
  const uintptr_t low = elem_bytes(dtype) - 1;
  if (!x || !out || !pos || (rot_dim > 0 && !turns) || (((uintptr_t)x | (uintptr_t)out) & low)) return PCM_ERR_ARG;
  if ((n_heads > 1 && ld_x_head < head_dim) || (n > 1 && ld_x < head_dim) || rows_overlap(n, n_heads, head_dim, ld_out, ld_out_head)) return PCM_ERR_ARG;
  if (x == out && (ld_x != ld_out || ld_x_head != ld_out_head)) return PCM_ERR_ARG;
  RotaryParams p = {};
  p.q = RotaryStream{x, ld_x, ld_x_head, out, ld_out, ld_out_head, n_heads};
  p.n = n; p.half = rot_dim / 2; p.dim = head_dim;
  p.turns = turns; p.amplitude = amplitude; p.inverse = (flags & GRPO_ROTARY_INVERSE) != 0; p.pos = pos;
  p.q_in_place = x == out;
  cudaStream_t s = (cudaStream_t)stream;
  prof_begin(PC_ELEM, s);
  const int rc = dtype == GRPO_BF16 ? launch_rotary<__nv_bfloat16>(p, flags & GRPO_ROTARY_INTERLEAVED, s)
                                    : launch_rotary<float>(p, flags & GRPO_ROTARY_INTERLEAVED, s);
  prof_end(s, 3.0 * n * n_heads * rot_dim, 2.0 * n * n_heads * head_dim * elem_bytes(dtype));
  return rc;
}

// Whether the slots of a cache that is written share elements: each stride, from the least on, has to span what lies within it.
static bool slots_overlap(const grpo_kv_cache* c) {
  struct Dim { int64_t ld, n; } d[3] = {{c->ld_head, c->n_kv_heads}, {c->ld_slot, c->page_size}, {c->ld_page, c->n_pages}};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (d[j].ld > d[j + 1].ld) { const Dim t = d[j]; d[j] = d[j + 1]; d[j + 1] = t; }
  __int128 span = c->head_dim;
  for (const Dim& x : d) {
    if (x.n == 1) continue;                    // leads nowhere
    if (x.ld < span) return true;
    span += (__int128)x.ld * (x.n - 1);
  }
  return c->k == c->v;
}

extern "C" int grpo_rotary_cache(const grpo_kv_cache* cache, const grpo_kv_batch* batch, int32_t n_rows, const void* q, int64_t ld_q,
                                 int64_t ld_q_head, int32_t n_heads, const void* k, int64_t ld_k, int64_t ld_k_head, const void* v,
                                 int64_t ld_v, int64_t ld_v_head, int32_t rot_dim, const double* turns, float amplitude,
                                 const int32_t* pos, uint32_t flags, void* q_out, int64_t ld_q_out, int64_t ld_q_out_head,
                                 uint32_t* device_status, pcm_stream stream) {
  const int bad = kv_check(cache, batch, n_rows);
  if (bad != PCM_OK) return bad;
  const int dim = cache->head_dim, n_kv = cache->n_kv_heads;
  if (n_heads < 0 || rot_dim < 0 || !std::isfinite(amplitude) || (flags & ~GRPO_ROTARY_INTERLEAVED)) return PCM_ERR_ARG;
  if (dim > PCM_MAX_ROTARY_DIM || rot_dim % 2 || rot_dim > dim || n_heads > (1 << 16) || n_kv > (1 << 16)) return PCM_ERR_SHAPE;
  if (n_rows == 0 || batch->n_seq == 0) return PCM_OK;
  if (slots_overlap(cache)) return PCM_ERR_ARG;
  if (!k || !v || (rot_dim > 0 && !turns) || (n_heads > 0 && (!q || !q_out))) return PCM_ERR_ARG;
  const uintptr_t low = elem_bytes(cache->dtype) - 1;
  if (((uintptr_t)k | (uintptr_t)v | (n_heads ? (uintptr_t)q | (uintptr_t)q_out : 0)) & low) return PCM_ERR_ARG;
  if (n_kv > 1 && (ld_k_head < dim || ld_v_head < dim)) return PCM_ERR_ARG;
  if (n_rows > 1 && (ld_k < dim || ld_v < dim)) return PCM_ERR_ARG;
  if ((n_heads > 1 && ld_q_head < dim) || (n_heads > 0 && n_rows > 1 && ld_q < dim)) return PCM_ERR_ARG;
  if (n_heads > 0 && rows_overlap(n_rows, n_heads, dim, ld_q_out, ld_q_out_head)) return PCM_ERR_ARG;
  if (n_heads > 0 && q == q_out && (ld_q != ld_q_out || ld_q_head != ld_q_out_head)) return PCM_ERR_ARG;
  RotaryParams p = {};
  p.q = RotaryStream{q, ld_q, ld_q_head, q_out, ld_q_out, ld_q_out_head, n_heads};
  p.k = RotaryStream{k, ld_k, ld_k_head, cache->k, 0, cache->ld_head, n_kv};
  p.v = RotaryStream{v, ld_v, ld_v_head, cache->v, 0, cache->ld_head, n_kv};
  p.n = n_rows; p.half = rot_dim / 2; p.dim = dim;
  p.turns = turns; p.amplitude = amplitude; p.pos = pos;
  p.to_cache = 1;
  p.q_in_place = n_heads > 0 && q == q_out;
  p.cache = kv_view(cache, batch, n_rows, device_status);
  cudaStream_t s = (cudaStream_t)stream;
  prof_begin(PC_ELEM, s);
  const int rc = cache->dtype == GRPO_BF16 ? launch_rotary<__nv_bfloat16>(p, flags & GRPO_ROTARY_INTERLEAVED, s)
                                           : launch_rotary<float>(p, flags & GRPO_ROTARY_INTERLEAVED, s);
  prof_end(s, 3.0 * n_rows * (n_heads + n_kv) * rot_dim, 2.0 * n_rows * (n_heads + 2 * n_kv) * dim * elem_bytes(cache->dtype));
  return rc;
}
