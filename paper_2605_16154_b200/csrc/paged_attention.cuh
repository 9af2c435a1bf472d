// Attention over a paged cache: how its work is cut, shared by the kernels that do it.
//
// A unit is `unit_rows` rows of one sequence and one key-value head (a row is a new token and one of the query heads that
// share the key-value head; token-major) and the tiles of keys that some of them see.  All units' tiles form one line, in the
// order of sequences, row tiles, heads, keys.  Every worker (a block) takes an equal piece of that line, so that one long
// sequence or many short ones keep all SMs equally busy; borders that would cut off less than a few tiles of a unit move to
// its end.  A piece of a unit leaves the unnormalised sum of its values, its maximum and its sum of weights in the workspace,
// and the combining kernel joins a unit's pieces in the order of its keys: nothing depends on which block ran when.
#pragma once
#include <cuda.h>

#include "paged.cuh"

namespace pcm {
namespace pga {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

struct Piece;
struct AttnParams {
  KvView c;
  const void* q; long long ld_q, ld_q_head;
  void* out; long long ld_out, ld_out_head;
  float* lse;
  int n_heads, group;
  FastDiv div_group;
  float scale_log2;                            // scale log2(e): weights are powers of two
  int window, sinks;                           // window 0: everything before
  int unit_rows, row_shift;                    // rows of a unit: 2^row_shift
  int tile, tile_shift;                        // keys of a tile: 2^tile_shift
  int over_rows, up_to_rows;                   // this kernel's sequences: over_rows < new tokens * group <= up_to_rows
  int workers, min_share;                      // pieces of the line; tiles of a piece at least
  long long* prefix;                           // [n_seq + 1] tiles ahead of each sequence; NULL: every block finds them itself
  int4* jobs;                                  // [workers] unit that a worker began and left open: sequence, row tile, head, last worker (-1: none)
  Piece* pieces;                               // [workers]
  int* redo;                                   // [workers] 1: a row of a whole unit is not finite although its weights are
  float* part;                                 // [2 workers][unit_rows][head_dim], then [2 workers][unit_rows] maxima and sums
  float2* part_ml;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A sequence's rows as this kernel sees them: none where another kernel takes the sequence.
__device__ __forceinline__ SeqSpan attn_span(const AttnParams& p, int s, bool report) {
  SeqSpan sp = seq_span(p.c, s, report);
  const long long rows = (long long)sp.fresh * p.group;
  if (rows <= p.over_rows || rows > p.up_to_rows) sp.fresh = 0;
  return sp;
}
__device__ __forceinline__ int row_tiles(const AttnParams& p, const SeqSpan& sp) {
  return (sp.fresh * p.group + p.unit_rows - 1) >> p.row_shift;
}

// The tiles that the rows of row tile qt see: tile i of the unit is tile i of the sequence below `first_tiles` and tile
// i + skip from there on.  Keys at or behind `end`, and from `sinks` up to `low`, are seen by none of them.
struct UnitSpan { int tiles, first_tiles, skip, end, low; };
__device__ __forceinline__ UnitSpan unit_span(const AttnParams& p, const SeqSpan& sp, int qt) {
  const int r0 = qt * p.unit_rows, r1 = min(r0 + p.unit_rows, sp.fresh * p.group) - 1, first = sp.len - sp.fresh;
  const int p0 = first + fast_div(r0, p.div_group), p1 = first + fast_div(r1, p.div_group);
  UnitSpan u;
  u.end = p1 >= 0 ? p1 + 1 : 0;
  u.low = p.window > 0 && p0 >= p.window ? p0 - p.window + 1 : 0;
  const int all = (u.end + p.tile - 1) >> p.tile_shift, from = u.low >> p.tile_shift;
  const int st = (min(p.sinks, u.end) + p.tile - 1) >> p.tile_shift;
  if (st >= from) {
    u.first_tiles = 0; u.skip = 0; u.tiles = max(1, all);          // a unit that sees nothing still writes its zeros
  } else {
    u.first_tiles = st; u.skip = from - st; u.tiles = all - u.skip;
  }
  return u;
}
__device__ __forceinline__ bool unit_sees(const AttnParams& p, const UnitSpan& u, int key) {
  return key < u.end && (key >= u.low || key < p.sinks);
}
__device__ __forceinline__ bool row_sees(const AttnParams& p, int pos, int key) {
  return key <= pos && (p.window == 0 || key > pos - p.window || key < p.sinks);
}

// A place on the line.
struct Cursor {
  int s, qt, head, at, nqt;                    // sequence, row tile, key-value head, tile; row tiles of the sequence
  SeqSpan sp;
  UnitSpan u;
  __device__ void enter_sequence(const AttnParams& p) {            // the next sequence with rows, from s on
    for (;; ++s) {
      if (s >= p.c.n_seq) { nqt = 0; return; }
      sp = attn_span(p, s, false);
      nqt = row_tiles(p, sp);
      if (nqt > 0) return;
    }
  }
  __device__ void next_unit(const AttnParams& p) {
    at = 0;
    if (++head < p.c.n_kv) return;
    head = 0;
    if (++qt >= nqt) {
      qt = 0; ++s;
      enter_sequence(p);
      if (nqt == 0) return;
    }
    u = unit_span(p, sp, qt);
  }
};

__device__ __forceinline__ long long line_share(const AttnParams& p, long long total) {
  const long long even = (total + p.workers - 1) / p.workers;
  return even > p.min_share ? even : p.min_share;
}
// A border at tile `at` of a unit of `tiles`: -at moves it to the unit's start, tiles - at to its end, 0 leaves it.
__device__ __forceinline__ int border_shift(const AttnParams& p, long long share, int at, int tiles) {
  const int slack = (int)min(1ll << 20, max((long long)(p.min_share + 1) / 2, share >> 6));
  if (at <= slack && at <= tiles - at) return -at;
  return tiles - at <= slack ? tiles - at : 0;
}

// Where border `i` of the line falls; called by a whole warp.  Returns the tiles ahead of it.
__device__ inline long long find_border(const AttnParams& p, const long long* prefix, int i, long long share, long long total, Cursor& c) {
  const int lane = threadIdx.x & 31;
  const long long x = share * i;
  if (x >= total) { c.s = p.c.n_seq; c.qt = c.head = c.at = c.nqt = 0; return total; }
  int lo = 0, hi = p.c.n_seq - 1;              // the sequence with prefix[s] <= x < prefix[s + 1]
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid + 1] > x) hi = mid; else lo = mid + 1;
  }
  c.s = lo;
  c.sp = attn_span(p, lo, false);
  c.nqt = row_tiles(p, c.sp);
  long long y = x - prefix[lo];
  for (int base = 0;; base += 32) {
    const int qt = base + lane;
    long long sum = qt < c.nqt ? (long long)unit_span(p, c.sp, qt).tiles * p.c.n_kv : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long t = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += t;
    }
    const unsigned over = __ballot_sync(0xffffffffu, sum > y);
    if (over || base + 32 >= c.nqt) {
      const int at = over ? __ffs(over) - 1 : 0;
      const long long before = __shfl_sync(0xffffffffu, sum, at > 0 ? at - 1 : 0);
      c.qt = base + at;
      if (at > 0) y -= before;
      break;
    }
    y -= __shfl_sync(0xffffffffu, sum, 31);
  }
  c.u = unit_span(p, c.sp, c.qt);
  c.head = y >> 31 ? (int)(y / c.u.tiles) : (int)y / c.u.tiles;     // (y is below the tiles of one row tile: all but always short)
  c.at = (int)(y - (long long)c.head * c.u.tiles);
  const int shift = border_shift(p, share, c.at, c.u.tiles);
  const bool to_end = shift > 0;
  c.at += shift;
  if (to_end) c.next_unit(p);
  return x + shift;
}

// The last worker that holds a piece of the unit which covers [first, first + tiles) of the line, worker w its first.
__device__ inline int last_worker(const AttnParams& p, int w, long long share, long long first, int tiles) {
  int e = w;
  for (;;) {
    const long long x = share * (e + 1) - first;                   // border e + 1, from the unit's start
    if (x >= tiles || x + border_shift(p, share, (int)x, tiles) >= tiles || e + 1 >= p.workers) return e;
    ++e;
  }
}

// Row r of row tile qt: its token's row in the call and position, and its query head.
struct RowPlace { long long row; int pos, head; bool valid; };
__device__ __forceinline__ RowPlace row_place(const AttnParams& p, const SeqSpan& sp, int qt, int kv_head, int r) {
  RowPlace x;
  const int R = qt * p.unit_rows + r;          // rows of a sequence are counted in 31 bits, and a unit more
  x.valid = R < sp.fresh * p.group;
  const int t = x.valid ? fast_div(R, p.div_group) : 0;
  x.row = sp.row0 + t;
  x.head = kv_head * p.group + (R - t * p.group);
  x.pos = x.valid ? sp.len - sp.fresh + t : -1;
  return x;
}

// First element of the slot of token `key` for a key-value head; -1 where the table names no page of the cache.
__device__ __forceinline__ long long slot_offset(const KvView& c, int s, int key, int head) {
  const int at = fast_div(key, c.div_page);
  const int page = c.table[s * c.ld_table + at];
  if (page < 0 || page >= c.n_pages) { kv_report(c, STATUS_BAD_PAGE); return -1; }
  return page * c.ld_page + (key - at * c.page_size) * c.ld_slot + head * c.ld_head;
}

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float& d, float x) { d = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16& d, float x) { d = __float2bfloat16_rn(x); }

// A zero weight times an infinity or a NaN is a NaN, so a value that one row does not see can reach it through the product of
// its tile.  A row whose values are not finite although the sum of its weights is gets formed once more, by a warp, key by key
// and without the keys it does not see (the kernels report it in `redo`, the joining kernel mends it).  Lane i holds columns
// i, i + 32, ..; returns the log-sum-exp.
template <typename T, int DH>
__device__ inline float exact_row(const AttnParams& p, int s, int kv_head, const UnitSpan& u, const RowPlace& x, float (&o)[DH / 32]) {
  const int lane = threadIdx.x & 31;
  const T* q = (const T*)p.q + x.row * p.ld_q + x.head * p.ld_q_head;
  float qv[DH / 32], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) { qv[i] = as_float(q[lane + 32 * i]); o[i] = 0.f; }
  for (int t = 0; t < u.tiles; ++t) {
    const int base = (t < u.first_tiles ? t : t + u.skip) * p.tile;
    for (int key = base; key < base + p.tile; ++key) {
      if (!row_sees(p, x.pos, key)) continue;
      const long long at = slot_offset(p.c, s, key, kv_head);
      float z = 0.f, v[DH / 32];
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) {
        const float k = at >= 0 ? as_float(((const T*)p.c.k)[at + lane + 32 * i]) : 0.f;
        v[i] = at >= 0 ? as_float(((const T*)p.c.v)[at + lane + 32 * i]) : 0.f;
        z = fmaf(qv[i], k, z);
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
      if (z == -INFINITY) continue;            // weighs nothing, and is no reference
      if (z > m) {
        const float f = ex2((m - z) * p.scale_log2);
        m = z;
        l *= f;
#pragma unroll
        for (int i = 0; i < DH / 32; ++i) o[i] *= f;
      }
      const float w = ex2((z - m) * p.scale_log2);
      l += w;
      if (w == 0.f) continue;
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) o[i] = fmaf(w, v[i], o[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) o[i] = l == 0.f ? 0.f : o[i] / l;
  return l == 0.f ? -INFINITY : fmaf(m, p.scale_log2, log2f(l)) * LN2;
}

// One worker's piece of the line.
struct Piece { Cursor c; long long left, share, ahead; };          // tiles left of the piece; tiles ahead of the cursor
// Tiles ahead of every sequence, by a whole block; `room`: LINE_ROOM bytes of shared memory.
constexpr int LINE_ROOM = 34 * 8 + 1024 * 4;
__device__ inline void line_prefix(const AttnParams& p, long long* prefix, void* room, bool report) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = (int)blockDim.x >> 5;
  long long* sums = (long long*)room;          // one a warp; the carry; how many sequences are listed
  long long* carry = sums + 32;
  int* listed = (int*)(sums + 33);
  int* list = (int*)(sums + 34);               // sequences of many row tiles: a warp each
  if (tid == 0) { *carry = 0; prefix[0] = 0; *listed = 0; }
  for (int base = 0; base < p.c.n_seq; base += (int)blockDim.x) {
    __syncthreads();
    const int s = base + tid;
    if (s < p.c.n_seq) {
      const SeqSpan sp = attn_span(p, s, report);
      const int nqt = row_tiles(p, sp);
      long long sum = 0;
      if (nqt <= 2)
        for (int qt = 0; qt < nqt; ++qt) sum += unit_span(p, sp, qt).tiles;
      else
        list[atomicAdd(listed, 1)] = s;        // in any order: each writes its own sequence's sum
      prefix[s + 1] = sum * p.c.n_kv;
    }
    __syncthreads();
    for (int i = warp; i < *listed; i += warps) {
      const SeqSpan sp = attn_span(p, list[i], false);
      const int nqt = row_tiles(p, sp);
      long long sum = 0;
      for (int qt = lane; qt < nqt; qt += 32) sum += unit_span(p, sp, qt).tiles;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (lane == 0) prefix[list[i] + 1] = sum * p.c.n_kv;
    }
    __syncthreads();
    long long sum = s < p.c.n_seq ? prefix[s + 1] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long t = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += t;
    }
    if (lane == 31) sums[warp] = sum;
    __syncthreads();
    long long before = *carry;
    for (int w = 0; w < warp; ++w) before += sums[w];
    if (s < p.c.n_seq) prefix[s + 1] = before + sum;
    __syncthreads();
    if (tid == (int)blockDim.x - 1) { *carry = before + sum; *listed = 0; }
  }
  __syncthreads();
}

// Sequences and row tiles (as the host can bound them) up to which every block finds its piece from the lengths: a launch and
// the reads of its results less (a step of one sequence: 12 us, 16 with them).
constexpr int SELF_PLANNED = 1024;
constexpr int SELF_BYTES = (SELF_PLANNED + 1) * 8 + LINE_ROOM;

// The block's piece of the line, from the plan's results or from the lengths; `scratch`: SELF_BYTES of shared memory.  Ends
// with a barrier of the block.
__device__ inline void block_piece(const AttnParams& p, void* scratch, Piece* piece) {
  const long long* prefix = p.prefix;
  if (!prefix) {
    long long* own = (long long*)scratch;
    line_prefix(p, own, own + SELF_PLANNED + 1, blockIdx.x == 0);
    prefix = own;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long total = prefix[p.c.n_seq], share = line_share(p, total);
  if (warp < 2) {                              // a warp for either border
    Cursor c;
    const long long x = find_border(p, prefix, (int)blockIdx.x + warp, share, total, c);
    if (lane == 0) {
      if (warp == 0) { piece->c = c; piece->ahead = x; piece->share = share; }
      else piece->left = x;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) piece->left -= piece->ahead;
  __syncthreads();
}

// Launches of the kernels on a line that is planned (workers, unit_rows and tile set).
bool page_map(CUtensorMap* tm, const void* base, const KvView& c, int dh, int box_cols, int box_rows);
int attn_rows_tile(int dh);
int launch_rows_bf16(const AttnParams& p, int dh, cudaStream_t s);
int attn_chunk_rows();
int attn_chunk_tile();
int launch_chunk_bf16(const AttnParams& p, int dh, cudaStream_t s);              // head dims 64 and 128

}  // namespace pga
}  // namespace pcm
