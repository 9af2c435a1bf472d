// The vocabulary ends of a policy: embedding lookup and its gradient, log-probabilities of given tokens from
// logits (with entropy, log-sum-exp and the top alternatives) and their gradient.  All of it is bound by HBM on
// large batches and by latency on single-token calls.
#include <cmath>

#include "async_ptx.cuh"
#include "internal.h"
#include "vocab.cuh"

namespace pcm {

// ------------------------------------------------------------------------------------------------
// 16-byte vectors of T, unpacked to fp32
// ------------------------------------------------------------------------------------------------
template <typename T> struct Vec16;
template <> struct Vec16<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[4]) {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Vec16<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// ------------------------------------------------------------------------------------------------
// Embedding lookup: out[i] = round(scale * table[tok[i]]); rows of a token outside [0, vocab) are zero.
// Bound by HBM (each distinct row read once, every output row written once); a block holds 256 / tpr rows, tpr
// threads walk one row in 16-byte steps, four loads in flight each.
// ------------------------------------------------------------------------------------------------
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
embed_kernel(const T* __restrict__ table, long long ld_table, int vocab, int d, const int* __restrict__ tok, int n, float scale,
             T* __restrict__ out, long long ld_out, unsigned* status, int tpr_log2) {
  const int tpr = 1 << tpr_log2;
  const long long row = ((long long)blockIdx.x << (8 - tpr_log2)) + (threadIdx.x >> tpr_log2);
  if (row >= n) return;
  const int lane = threadIdx.x & (tpr - 1);
  const int t = tok[row];
  const bool live = t >= 0 && t < vocab;
  if (t >= vocab && lane == 0 && status) atomicOr(status, STATUS_BAD_TOKEN);
  const T* src = table + (long long)(live ? t : 0) * ld_table;
  T* dst = out + row * ld_out;
  if constexpr (VEC) {
    using V = Vec16<T>;
    const int nv = d / V::N;
    const uint4* s4 = reinterpret_cast<const uint4*>(src);
    uint4* d4 = reinterpret_cast<uint4*>(dst);
    for (int v0 = lane; v0 < nv; v0 += 4 * tpr) {
      uint4 r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int v = v0 + u * tpr;
        r[u] = make_uint4(0, 0, 0, 0);
        if (live && v < nv) r[u] = __ldg(s4 + v);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int v = v0 + u * tpr;
        float f[V::N];
        V::unpack(r[u], f);
#pragma unroll
        for (int e = 0; e < V::N; ++e) f[e] *= scale;
        if (v < nv) __stcs(d4 + v, live ? V::pack(f) : make_uint4(0, 0, 0, 0));
      }
    }
  } else {
    for (int c = lane; c < d; c += tpr) dst[c] = live ? from_f32<T>(as_f32(src[c]) * scale) : from_f32<T>(0.f);
  }
}

// ------------------------------------------------------------------------------------------------
// Gradient of the embedding: grad[v] (+)= scale * sum over {i : tok[i] = v} of dout[i], in fp32 and in ascending i.
//   1. embed_sort_kernel: (token, position) pairs into token order by a stable radix sort inside one cluster;
//   2. embed_sum_kernel: tiles of `rows` sorted pairs, each summed in order; a token that lies inside one tile is
//      final, one that crosses tiles leaves a partial sum per tile; rows of absent tokens are written as zero;
//   3. embed_join_kernel: the partial sums of the crossing tokens, in tile order.
// No floating-point atomics: the same inputs give the same bits.  Bound by HBM: dout once, grad once.
// ------------------------------------------------------------------------------------------------
constexpr int ES_THREADS = 1024, ES_WARPS = ES_THREADS / 32, ES_BINS = 256, ES_MAX_RANKS = 8, ES_BATCH = 8;

struct EmbedPlan {
  int n, vocab, d;
  int rows, tiles, dpad;                      // sorted pairs per tile, tiles, floats per partial row
  uint2* buf[2];                              // (token, position) pairs
  uint8_t* present;                           // [vocab] 1 where a token occurs
  int* n_jobs; int* jobs;                     // tiles in which a crossing token begins
  float* part;                                // [tiles][2][dpad]: of a token that began before the tile, of one that goes on behind it
  const uint2* sorted;                        // the buffer that the last pass of the sort fills
};

struct EmbedSortSmem {
  unsigned count[ES_WARPS][ES_BINS];
  unsigned total[ES_BINS];
  unsigned base[ES_BINS];
  unsigned warp_sum[ES_BINS / 32];
};

__device__ __forceinline__ unsigned ld_shared_cluster(uint32_t addr) {
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

__global__ void __launch_bounds__(ES_THREADS)
embed_sort_kernel(const int* __restrict__ tok, const EmbedPlan pl, int ranks, int passes, int bits, unsigned* status) {
  __shared__ EmbedSortSmem sm;
  const int rank = ranks == 1 ? 0 : (int)cluster_ctarank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lo = (int)((long long)pl.n * rank / ranks), hi = (int)((long long)pl.n * (rank + 1) / ranks);
  const int wlo = lo + (int)((long long)(hi - lo) * warp / ES_WARPS), whi = lo + (int)((long long)(hi - lo) * (warp + 1) / ES_WARPS);
  for (long long i = (long long)rank * ES_THREADS + threadIdx.x; i < (pl.vocab + 15) / 16; i += (long long)ranks * ES_THREADS)
    reinterpret_cast<uint4*>(pl.present)[i] = make_uint4(0, 0, 0, 0);
  if (rank == 0 && threadIdx.x == 0) *pl.n_jobs = 0;
  const unsigned mask = (1u << bits) - 1u;
  for (int pass = 0; pass < passes; ++pass) {
    const uint2* src = (pass & 1) ? pl.buf[0] : pl.buf[1];
    uint2* dst = (pass & 1) ? pl.buf[1] : pl.buf[0];
    const int shift = pass * bits;
    const bool last = pass == passes - 1;
    // the pair at sorted-so-far position i; tokens outside the vocabulary take the key behind its last one
    auto fetch = [&](int i, uint2& kv) {
      if (pass == 0) {
        const int t = tok[i];
        kv = make_uint2(t >= 0 && t < pl.vocab ? (unsigned)t : (unsigned)pl.vocab, (unsigned)i);
        return t >= pl.vocab;
      }
      kv = __ldcg(src + i);
      return false;
    };
    for (int i = threadIdx.x; i < ES_WARPS * ES_BINS; i += ES_THREADS) (&sm.count[0][0])[i] = 0;
    __syncthreads();
    bool bad = false;
    for (int b = wlo; b < whi; b += 32 * ES_BATCH) {
      uint2 kv[ES_BATCH];
#pragma unroll
      for (int u = 0; u < ES_BATCH; ++u) {
        const int i = b + u * 32 + lane;
        if (i < whi) bad |= fetch(i, kv[u]);
      }
#pragma unroll
      for (int u = 0; u < ES_BATCH; ++u) {
        const bool in = b + u * 32 + lane < whi;
        const unsigned dig = in ? (kv[u].x >> shift) & mask : 0xFFFFFFFFu;
        const unsigned same = __match_any_sync(0xffffffffu, dig);
        if (in && lane == __ffs(same) - 1) sm.count[warp][dig] += __popc(same);
        __syncwarp();
      }
    }
    if (bad && status) atomicOr(status, STATUS_BAD_TOKEN);
    __syncthreads();
    // per digit: where each warp's pairs begin among this block's
    if (threadIdx.x < ES_BINS) {
      unsigned run = 0;
#pragma unroll 8
      for (int w = 0; w < ES_WARPS; ++w) {
        const unsigned k = sm.count[w][threadIdx.x];
        sm.count[w][threadIdx.x] = run;
        run += k;
      }
      sm.total[threadIdx.x] = run;
    }
    __syncthreads();
    if (ranks > 1) cluster_sync_all();
    // per digit: pairs of smaller digits in all blocks, then of this digit in the blocks before this one
    unsigned before = 0, all = 0, incl = 0;
    if (threadIdx.x < ES_BINS) {
      const uint32_t mine = smem_u32(&sm.total[threadIdx.x]);
      for (int r = 0; r < ranks; ++r) {
        const unsigned k = ranks == 1 ? sm.total[threadIdx.x] : ld_shared_cluster(mapa_shared(mine, (uint32_t)r));
        all += k;
        before += r < rank ? k : 0;
      }
      incl = all;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const unsigned o = __shfl_up_sync(0xffffffffu, incl, off);
        incl += lane >= off ? o : 0;
      }
      if (lane == 31) sm.warp_sum[warp] = incl;
    }
    __syncthreads();
    if (threadIdx.x < ES_BINS) {
      unsigned start = incl - all;
      for (int w = 0; w < warp; ++w) start += sm.warp_sum[w];
      sm.base[threadIdx.x] = start + before;
    }
    __syncthreads();
    for (int b = wlo; b < whi; b += 32 * ES_BATCH) {
      uint2 kv[ES_BATCH];
#pragma unroll
      for (int u = 0; u < ES_BATCH; ++u) {
        const int i = b + u * 32 + lane;
        if (i < whi) fetch(i, kv[u]);
      }
#pragma unroll
      for (int u = 0; u < ES_BATCH; ++u) {
        const bool in = b + u * 32 + lane < whi;
        const unsigned dig = in ? (kv[u].x >> shift) & mask : 0xFFFFFFFFu;
        const unsigned same = __match_any_sync(0xffffffffu, dig);
        unsigned at = 0;
        if (in) at = sm.base[dig] + sm.count[warp][dig] + __popc(same & ((1u << lane) - 1u));
        __syncwarp();
        if (in) {
          if (lane == __ffs(same) - 1) sm.count[warp][dig] += __popc(same);
          dst[at] = kv[u];
          if (last && kv[u].x < (unsigned)pl.vocab) pl.present[kv[u].x] = 1;
        }
        __syncwarp();
      }
    }
    if (ranks > 1) cluster_sync_all();        // the pairs are in place, the digit totals have been read
    else __syncthreads();
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(128)
embed_sum_kernel(const T* __restrict__ dout, long long ld, const EmbedPlan pl, float scale, float* __restrict__ grad, int accumulate,
                 int ct_log2, int slabs, int tile_blocks) {
  constexpr int N = VEC ? Vec16<T>::N : 1;
  if ((int)blockIdx.x >= tile_blocks) {       // rows of absent tokens, 32 per block
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int k = 0; k < 8; ++k) {
      const long long v = (long long)(blockIdx.x - tile_blocks) * 32 + k * 4 + warp;
      if (v >= pl.vocab || pl.present[v]) continue;
      float* g = grad + v * pl.d;
      if (VEC) {
        for (int c = lane * 4; c < pl.d; c += 128) __stcs(reinterpret_cast<float4*>(g + c), make_float4(0.f, 0.f, 0.f, 0.f));
      } else {
        for (int c = lane; c < pl.d; c += 32) g[c] = 0.f;
      }
    }
    return;
  }
  const int slab = blockIdx.x % slabs;
  const int tile = ((blockIdx.x / slabs) << (7 - ct_log2)) + (threadIdx.x >> ct_log2);
  const int col = (slab << (ct_log2)) * N + (threadIdx.x & ((1 << ct_log2) - 1)) * N;
  if (tile >= pl.tiles || col >= pl.d) return;
  const uint2* pair = pl.sorted;
  const int lo = tile * pl.rows, hi = min(lo + pl.rows, pl.n);
  const unsigned before = lo > 0 ? pair[lo - 1].x : 0xFFFFFFFFu, behind = hi < pl.n ? pair[hi].x : 0xFFFFFFFFu;
  unsigned cur = pair[lo].x;
  bool first = true;
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  auto put = [&](float* dst, float f, bool add) {
#pragma unroll
    for (int e = 0; e < N; e += (N >= 4 ? 4 : 1)) {
      if constexpr (N >= 4) {
        float4 o = make_float4(acc[e] * f, acc[e + 1] * f, acc[e + 2] * f, acc[e + 3] * f);
        float4* q = reinterpret_cast<float4*>(dst + e);
        if (add) { const float4 w = *q; o.x += w.x; o.y += w.y; o.z += w.z; o.w += w.w; }
        *q = o;
      } else {
        dst[e] = add ? dst[e] + acc[e] * f : acc[e] * f;
      }
    }
  };
  auto flush = [&](bool goes_on) {
    if (cur >= (unsigned)pl.vocab) return;
    const bool began_before = first && cur == before;
    if (began_before) {
      put(pl.part + ((long long)tile * 2) * pl.dpad + col, 1.f, false);
    } else if (goes_on) {
      put(pl.part + ((long long)tile * 2 + 1) * pl.dpad + col, 1.f, false);
      if (col == 0) pl.jobs[atomicAdd(pl.n_jobs, 1)] = tile;
    } else {
      put(grad + (long long)cur * pl.d + col, scale, accumulate != 0);
    }
  };
  for (int i0 = lo; i0 < hi; i0 += 8) {
    uint2 kv[8];
    uint4 raw[8];
    float one[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) kv[u] = i0 + u < hi ? pair[i0 + u] : make_uint2(0xFFFFFFFFu, 0u);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (kv[u].x < (unsigned)pl.vocab) {
        const T* q = dout + (long long)kv[u].y * ld + col;
        if constexpr (VEC) raw[u] = __ldcs(reinterpret_cast<const uint4*>(q));
        else one[u] = as_f32(*q);
      }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (i0 + u >= hi) break;
      if (kv[u].x != cur) {
        flush(false);
        cur = kv[u].x;
        first = false;
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.f;
      }
      if (cur < (unsigned)pl.vocab) {
        if constexpr (VEC) {
          float f[N];
          Vec16<T>::unpack(raw[u], f);
#pragma unroll
          for (int e = 0; e < N; ++e) acc[e] += f[e];
        } else {
          acc[0] += one[u];
        }
      }
    }
  }
  flush(cur == behind);
}

// One warp per crossing token and 128 columns; a token over more than 16 tiles is shared by the block's eight warps.
__global__ void __launch_bounds__(256)
embed_join_kernel(const EmbedPlan pl, float scale, float* __restrict__ grad, int accumulate) {
  __shared__ float4 sum[8][32];
  __shared__ int span[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_jobs = *pl.n_jobs;
  if ((int)blockIdx.x * 8 >= n_jobs) return;
  const uint2* pair = pl.sorted;
  const int col = (blockIdx.y * 32 + lane) * 4;
  const int job = blockIdx.x * 8 + warp;
  // tiles after the first one that the token reaches into
  int more = 0;
  if (job < n_jobs) {
    const int t = pl.jobs[job];
    const unsigned key = pair[(long long)(t + 1) * pl.rows - 1].x;
    for (int base = t + 1;; base += 32) {
      const int u = base + lane;
      const bool on = u < pl.tiles && pair[(long long)u * pl.rows].x == key;
      const unsigned m = __ballot_sync(0xffffffffu, on);
      if (m != 0xffffffffu) { more += __ffs(~m) - 1; break; }
      more += 32;
    }
  }
  if (lane == 0) span[warp] = more;
  __syncthreads();
  auto add_tiles = [&](float4& a, int t, int lo, int hi) {      // partial sums of tiles t + lo .. t + hi - 1 (0: the first tile)
#pragma unroll 4
    for (int k = lo; k < hi; ++k) {
      const float* q = pl.part + ((long long)(t + k) * 2 + (k == 0 ? 1 : 0)) * pl.dpad + col;
      const float4 w = *reinterpret_cast<const float4*>(q);
      a.x += w.x; a.y += w.y; a.z += w.z; a.w += w.w;
    }
  };
  auto finish = [&](const float4& a, int t) {
    const unsigned key = pair[(long long)(t + 1) * pl.rows - 1].x;
    float* g = grad + (long long)key * pl.d + col;
    const float v[4] = {a.x * scale, a.y * scale, a.z * scale, a.w * scale};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < pl.d) g[e] = accumulate ? g[e] + v[e] : v[e];
  };
  const bool in = col < pl.d;                 // partial rows are padded to a multiple of four
  if (job < n_jobs && span[warp] <= 16 && in) {
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    const int t = pl.jobs[job];
    add_tiles(a, t, 0, span[warp] + 1);
    finish(a, t);
  }
  for (int j = 0; j < 8; ++j) {
    if (span[j] <= 16) continue;              // the same for the whole block
    const int t = pl.jobs[blockIdx.x * 8 + j], len = span[j] + 1;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    if (in) add_tiles(a, t, len * warp / 8, len * (warp + 1) / 8);
    sum[warp][lane] = a;
    __syncthreads();
    if (warp == 0 && in) {
      for (int w = 1; w < 8; ++w) {
        const float4 b = sum[w][lane];
        a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
      }
      finish(a, t);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------
// Log-probabilities of given tokens from logits.
// ------------------------------------------------------------------------------------------------
// Whole numbers in the order of the floats they stand for: -0 and +0 are one value, a NaN of either sign is above all.
__device__ __forceinline__ unsigned order_of(float z) {
  if (z != z) return 0xFFFFFFFFu;
  const unsigned u = __float_as_uint(z + 0.f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float float_of_order(unsigned o) {
  if (o == 0xFFFFFFFFu) return __uint_as_float(0x7FFFFFFFu);
  return __uint_as_float((o & 0x80000000u) ? (o ^ 0x80000000u) : ~o);
}

struct LogpParams {
  const void* logits; long long ld;
  int M, V;
  const int* tok;
  float inv_t;
  int top;
  float* logp; float* entropy; float* lse;
  int* top_id; float* top_logp;
  unsigned* status;
};

template <typename T>
__device__ __forceinline__ void part_add(VocabStat& st, const float (&v)[Vec16<T>::N], float c) {
  constexpr int N = Vec16<T>::N;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float t = fmaxf((v[e] - st.m) * c, -1000.f);
    const float x = ex2(t);
    st.s += x;
    st.w += x * t;
  }
}

// A row (or a cluster rank's share of it) as 16-byte vectors plus up to N - 1 single elements before and after.
template <typename T>
struct RowShare {
  const T* p;
  int head, v_lo, v_hi, tail;                 // elements before the first vector; vectors of this share; first element after
  int V;
  bool has_head, has_tail;
  __device__ RowShare(const T* row, int V_, int rank, int ranks) : p(row), V(V_) {
    constexpr int N = Vec16<T>::N;
    head = (int)(((16u - ((unsigned)(uintptr_t)row & 15u)) & 15u) / sizeof(T));
    if (head > V) head = V;
    const int nv = (V - head) / N;
    tail = head + nv * N;
    v_lo = (int)((long long)nv * rank / ranks);
    v_hi = (int)((long long)nv * (rank + 1) / ranks);
    has_head = rank == 0;
    has_tail = rank == ranks - 1;
  }
  __device__ __forceinline__ const uint4* vec(int v) const { return reinterpret_cast<const uint4*>(p + head) + v; }
  // the single element of thread `i` (head elements first, then the tail's), -1 when it has none
  __device__ __forceinline__ int single(int i) const {
    if (has_head && i < head) return i;
    i -= has_head ? head : 0;
    return (has_tail && i >= 0 && i < V - tail) ? tail + i : -1;
  }
};

constexpr int LP_MAX_TOP = PCM_MAX_TOP;
constexpr int LP_MAX_RANKS = 8;

// NT threads work on one row's share.  NT = 32: a warp per row, several rows per block.  Otherwise one block per share,
// `ranks` blocks of a cluster per row.
template <int NT> struct LogpSmem {
  static constexpr int CAP = NT == 32 ? 128 : 1024;
  unsigned long long cand[CAP];               // candidates of the top list: order_of(z) above, ~index below
  unsigned group_max[32];
  VocabStat part[32];
  int n_cand;
  unsigned long long best[NT == 32 ? 1 : LP_MAX_RANKS * LP_MAX_TOP];   // rank 0: the shares' own top lists
  VocabStat share[NT == 32 ? 1 : LP_MAX_RANKS];
};

template <int NT> __device__ __forceinline__ void row_sync() {
  if constexpr (NT == 32) __syncwarp(); else __syncthreads();
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT == 32 ? 256 : NT)
token_logp_kernel(const LogpParams p, int ranks) {
  using V16 = Vec16<T>;
  constexpr int N = V16::N, U = 4;
  constexpr int ROWS = NT == 32 ? 8 : 1;
  __shared__ LogpSmem<NT> smem_all[ROWS];
  LogpSmem<NT>& sm = smem_all[NT == 32 ? threadIdx.x >> 5 : 0];
  const int tid = NT == 32 ? threadIdx.x & 31 : threadIdx.x;
  const int lane = threadIdx.x & 31;
  const int rank = NT == 32 || ranks == 1 ? 0 : (int)cluster_ctarank();
  const long long row = NT == 32 ? (long long)blockIdx.x * ROWS + (threadIdx.x >> 5) : blockIdx.x / ranks;
  if (row >= p.M) return;                     // whole warps (NT = 32) only: the grid is exact otherwise
  const float c = p.inv_t * VOCAB_LOG2E;
  const int t = p.tok ? p.tok[row] : 0;
  const bool bad = p.tok && t >= p.V, skip = p.tok && (t < 0 || bad);
  const int top = p.top;
  if (skip) {                                 // the same for every thread of the row, every rank of its cluster
    if (rank == 0) {
      if (tid == 0) {
        if (bad && p.status) atomicOr(p.status, STATUS_BAD_TOKEN);
        if (p.logp) p.logp[row] = 0.f;
        if (p.entropy) p.entropy[row] = 0.f;
        if (p.lse) p.lse[row] = 0.f;
      }
      if (tid < top) { p.top_id[row * top + tid] = -1; p.top_logp[row * top + tid] = 0.f; }
    }
    return;
  }
  const RowShare<T> sh(reinterpret_cast<const T*>(p.logits) + row * p.ld, p.V, rank, ranks);
  if (tid == 0) sm.n_cand = 0;

  // ---- one pass over the share -------------------------------------------------------------------
  VocabStat st{-INFINITY, 0.f, 0.f};
  {
    const int e = sh.single(tid);
    if (e >= 0) {
      const float z = as_f32(sh.p[e]);
      st.m = z;
      const float x = z == -INFINITY ? 0.f : 1.f;
      st.s = x;
    }
  }
  for (int v0 = sh.v_lo + tid; v0 < sh.v_hi; v0 += U * NT) {
    uint4 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (v0 + u * NT < sh.v_hi) r[u] = __ldg(sh.vec(v0 + u * NT));
    float bm = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (v0 + u * NT < sh.v_hi) {
        float f[N];
        V16::unpack(r[u], f);
#pragma unroll
        for (int e = 0; e < N; ++e) bm = max_nan(bm, f[e]);
      }
    stat_raise(st, bm, c);
    if (st.m != -INFINITY) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * NT < sh.v_hi) {
          float f[N];
          V16::unpack(r[u], f);
          part_add<T>(st, f, c);
        }
    }
  }

  // ---- join the threads -----------------------------------------------------------------------------
  const unsigned own_max = order_of(st.m);    // -inf where the thread has no element: never above an element's
  if (top > 0) {
    unsigned g = own_max;
#pragma unroll
    for (int off = 1; off < NT / 32; off <<= 1) g = max(g, __shfl_xor_sync(0xffffffffu, g, off));
    if (tid % (NT / 32) == 0) sm.group_max[tid / (NT / 32)] = g;
  }
#pragma unroll
  for (int off = 16; off; off >>= 1) {
    VocabStat o;
    o.m = __shfl_xor_sync(0xffffffffu, st.m, off);
    o.s = __shfl_xor_sync(0xffffffffu, st.s, off);
    o.w = __shfl_xor_sync(0xffffffffu, st.w, off);
    st = stat_join(st, o, c);
  }
  if (lane == 0) sm.part[tid >> 5] = st;
  row_sync<NT>();
  if (NT > 32) {
    st = lane < NT / 32 ? sm.part[lane] : VocabStat{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      VocabStat o;
      o.m = __shfl_xor_sync(0xffffffffu, st.m, off);
      o.s = __shfl_xor_sync(0xffffffffu, st.s, off);
      o.w = __shfl_xor_sync(0xffffffffu, st.w, off);
      st = stat_join(st, o, c);
    }
  }

  // Every thread takes lane 0's result: the lanes join in different orders, and which lane writes a place of the top
  // list is decided by an atomic counter.
  st.m = __shfl_sync(0xffffffffu, st.m, 0);
  st.s = __shfl_sync(0xffffffffu, st.s, 0);
  st.w = __shfl_sync(0xffffffffu, st.w, 0);

  // ---- top list of the share ---------------------------------------------------------------------
  // The threads form 32 groups; the top-th largest of the groups' maxima is a value that at least `top` elements
  // reach.  Only threads whose own maximum reaches it read their elements again (from L2) and put those that do on a
  // list, whose members find their places by counting.  A list that overflows (many equal values, a mask that leaves
  // fewer than `top`) falls back to one search of the share for each place.
  int n = 0;
  bool overflow = false;
  if (top > 0) {
    const unsigned mine = sm.group_max[lane];
    int place = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const unsigned o = __shfl_sync(0xffffffffu, mine, j);
      place += (o > mine || (o == mine && j < lane)) ? 1 : 0;
    }
    const unsigned limit = __shfl_sync(0xffffffffu, mine, __ffs(__ballot_sync(0xffffffffu, place == top - 1)) - 1);
    if (own_max >= limit) {
      auto offer = [&](float z, int idx) {
        const unsigned o = order_of(z);
        if (o >= limit) {
          const int at = atomicAdd(&sm.n_cand, 1);
          if (at < LogpSmem<NT>::CAP) sm.cand[at] = ((unsigned long long)o << 32) | (0xFFFFFFFFu - (unsigned)idx);
        }
      };
      const int e = sh.single(tid);
      if (e >= 0) offer(as_f32(sh.p[e]), e);
      for (int v = sh.v_lo + tid; v < sh.v_hi; v += NT) {
        float f[N];
        V16::unpack(__ldg(sh.vec(v)), f);
#pragma unroll
        for (int k = 0; k < N; ++k) offer(f[k], sh.head + v * N + k);
      }
    }
    row_sync<NT>();
    n = sm.n_cand;
    overflow = n > LogpSmem<NT>::CAP;
  }
  auto search = [&](unsigned long long below) {          // largest key of the share under `below`, 0 when there is none
    unsigned long long best = 0;
    auto offer = [&](float z, int idx) {
      const unsigned long long key = ((unsigned long long)order_of(z) << 32) | (0xFFFFFFFFu - (unsigned)idx);
      if (key < below && key > best) best = key;
    };
    const int e = sh.single(tid);
    if (e >= 0) offer(as_f32(sh.p[e]), e);
    for (int v = sh.v_lo + tid; v < sh.v_hi; v += NT) {
      float f[N];
      V16::unpack(__ldg(sh.vec(v)), f);
#pragma unroll
      for (int k = 0; k < N; ++k) offer(f[k], sh.head + v * N + k);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      const unsigned long long o = __shfl_xor_sync(0xffffffffu, best, off);
      best = o > best ? o : best;
    }
    if (NT > 32) {
      __syncthreads();
      if (lane == 0) sm.cand[tid >> 5] = best;
      __syncthreads();
      best = 0;
      for (int i = 0; i < NT / 32; ++i) best = sm.cand[i] > best ? sm.cand[i] : best;
    }
    return best;
  };

  auto write_top = [&](const RowResult& res, int place, unsigned long long key) {
    p.top_id[row * top + place] = (int)(0xFFFFFFFFu - (unsigned)key);
    p.top_logp[row * top + place] = res.logp(float_of_order((unsigned)(key >> 32)));
  };
  auto write_row = [&](const RowResult& res) {
    if (p.tok && p.logp) p.logp[row] = res.logp(as_f32(sh.p[t]));
    if (p.entropy) p.entropy[row] = res.entropy;
    if (p.lse) p.lse[row] = res.lse;
  };
  if (NT == 32 || ranks == 1) {
    const RowResult res(st, p.inv_t);
    if (tid == 0) write_row(res);
    if (top > 0 && !overflow) {
      for (int i = tid; i < n; i += NT) {
        const unsigned long long key = sm.cand[i];
        int place = 0;
        for (int j = 0; j < n; ++j) place += sm.cand[j] > key ? 1 : 0;
        if (place < top) write_top(res, place, key);
      }
    } else if (top > 0) {
      unsigned long long below = ~0ull;
      for (int k = 0; k < top; ++k) {
        below = search(below);
        if (tid == 0) write_top(res, k, below);
      }
    }
    return;
  }
  if constexpr (NT > 32) {
    // ---- join the shares of a cluster on rank 0 ----
    cluster_sync_all();                       // rank 0 runs: its shared memory may be written
    const uint32_t share0 = mapa_shared(smem_u32(&sm.share[rank]), 0);
    const uint32_t best0 = mapa_shared(smem_u32(&sm.best[rank * LP_MAX_TOP]), 0);
    auto put = [&](int place, unsigned long long key) {
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(best0 + (uint32_t)place * 8u), "l"(key) : "memory");
    };
    if (tid == 0) {
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(share0), "f"(st.m) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(share0 + 4u), "f"(st.s) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(share0 + 8u), "f"(st.w) : "memory");
    }
    if (top > 0 && !overflow) {
      if (tid >= n && tid < top) put(tid, 0);           // a share with fewer elements than places
      for (int i = tid; i < n; i += NT) {
        const unsigned long long key = sm.cand[i];
        int place = 0;
        for (int j = 0; j < n; ++j) place += sm.cand[j] > key ? 1 : 0;
        if (place < top) put(place, key);
      }
    } else if (top > 0) {
      unsigned long long below = ~0ull;
      for (int k = 0; k < top; ++k) {
        below = below ? search(below) : 0;
        if (tid == 0) put(k, below);
      }
    }
    cluster_sync_all();
    if (rank != 0) return;
    st = sm.share[0];
    for (int r = 1; r < ranks; ++r) st = stat_join(st, sm.share[r], c);
    const RowResult res(st, p.inv_t);
    if (tid == 0) write_row(res);
    if (tid < ranks * LP_MAX_TOP && tid % LP_MAX_TOP < top) {
      const unsigned long long key = sm.best[tid];
      int place = 0;
      for (int r = 0; r < ranks; ++r)
        for (int k = 0; k < top; ++k) place += sm.best[r * LP_MAX_TOP + k] > key ? 1 : 0;
      if (key && place < top) write_top(res, place, key);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Gradient: d loss / d z_v = (1/T) (g (1[v = t] - p_v) - h p_v (log p_v + H)), g = d loss / d logp, h = d loss / d H.
// One read and one write of the logits; a thread reads what it writes, so dlogits may be the logits themselves.
// ------------------------------------------------------------------------------------------------
struct LogpBwdParams {
  const void* logits; long long ld;
  void* dlogits; long long ld_d;
  int M, V;
  const int* tok;
  const float* lse; const float* entropy; const float* dlogp; const float* dent;
  float inv_t;
  unsigned* status;
};

constexpr int LB_THREADS = 256;

template <typename T, bool VEC>
__global__ void __launch_bounds__(LB_THREADS)
token_logp_bwd_kernel(const LogpBwdParams p, int chunks) {
  using V16 = Vec16<T>;
  constexpr int N = V16::N, U = VEC ? 2 : 8;
  const long long row = blockIdx.x / chunks;
  const int chunk = blockIdx.x - (int)(row * chunks);
  const int t = p.tok[row];
  const float lse = p.lse[row];
  const bool live = t >= 0 && t < p.V && lse != -INFINITY;
  if (t >= p.V && chunk == 0 && threadIdx.x == 0 && p.status) atomicOr(p.status, STATUS_BAD_TOKEN);
  const float g = p.dlogp[row], h = p.dent ? p.dent[row] : 0.f;
  const float gt = g * p.inv_t, ht = h * p.inv_t, H = p.dent ? p.entropy[row] : 0.f;
  const T* z = reinterpret_cast<const T*>(p.logits) + row * p.ld;
  T* dz = reinterpret_cast<T*>(p.dlogits) + row * p.ld_d;
  auto slope = [&](float zv, int idx) { return vocab_slope(zv, p.inv_t, lse, H, gt, ht, idx == t); };
  if constexpr (VEC) {
    const int head = min(p.V, (int)(((16u - ((unsigned)(uintptr_t)z & 15u)) & 15u) / sizeof(T)));
    const int nv = (p.V - head) / N, tail = head + nv * N;
    const uint4* z4 = reinterpret_cast<const uint4*>(z + head);
    uint4* d4 = reinterpret_cast<uint4*>(dz + head);
    const int v0 = chunk * (LB_THREADS * U) + threadIdx.x;
    uint4 r[U];
    if (live) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * LB_THREADS < nv) r[u] = __ldcs(z4 + v0 + u * LB_THREADS);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v0 + u * LB_THREADS;
      if (v < nv) {
        uint4 o = make_uint4(0, 0, 0, 0);
        if (live) {
          float f[N];
          V16::unpack(r[u], f);
#pragma unroll
          for (int e = 0; e < N; ++e) f[e] = slope(f[e], head + v * N + e);
          o = V16::pack(f);
        }
        __stcs(d4 + v, o);
      }
    }
    if (chunk == 0) {
      const int i = threadIdx.x < head ? threadIdx.x : tail + threadIdx.x - head;
      if (threadIdx.x < head + (p.V - tail)) dz[i] = from_f32<T>(live ? slope(as_f32(z[i]), i) : 0.f);
    }
  } else {
    const int i0 = chunk * (LB_THREADS * U) + threadIdx.x;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * LB_THREADS;
      if (i < p.V) dz[i] = from_f32<T>(live ? slope(as_f32(z[i]), i) : 0.f);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
template <typename T>
static int launch_embed(const T* table, long long ld_table, int vocab, int d, const int* tok, int n, float scale, T* out,
                        long long ld_out, unsigned* status, cudaStream_t s) {
  constexpr int N = Vec16<T>::N;
  const bool vec = !(((uintptr_t)table | (uintptr_t)out) & 15) && d % N == 0 && ld_table % N == 0 && ld_out % N == 0;
  const int steps = vec ? d / N : d;
  int lg = 0;                                 // threads per row: a power of two, four steps each once the rows fill the GPU
  const long long per = (long long)n * steps / 4 >= 256ll * sm_count() * 2 ? 4 : 1;
  while (lg < 8 && (per << lg) < steps) ++lg;
  const long long blocks = ((long long)n + (256 >> lg) - 1) >> (8 - lg);
  if (vec) embed_kernel<T, true><<<(unsigned)blocks, 256, 0, s>>>(table, ld_table, vocab, d, tok, n, scale, out, ld_out, status, lg);
  else embed_kernel<T, false><<<(unsigned)blocks, 256, 0, s>>>(table, ld_table, vocab, d, tok, n, scale, out, ld_out, status, lg);
  PCM_LAUNCH_CHECK();
  return PCM_OK;
}

// Sorted pairs per tile: 64 once that leaves two blocks for each SM, fewer for short batches.
static int embed_tile_rows(int n) { return n >= 64 * 296 ? 64 : 16; }

static size_t embed_plan(EmbedPlan& pl, int n, int vocab, int d, void* ws) {
  pl.n = n; pl.vocab = vocab; pl.d = d;
  pl.rows = embed_tile_rows(n);
  pl.tiles = ceil_div(n, pl.rows);
  pl.dpad = (d + 3) / 4 * 4;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* q = (unsigned char*)ws + off;
    off += (bytes + 255) / 256 * 256;
    return q;
  };
  pl.buf[0] = (uint2*)take((size_t)n * 8);
  pl.buf[1] = (uint2*)take((size_t)n * 8);
  pl.present = (uint8_t*)take((size_t)vocab);
  pl.n_jobs = (int*)take(4);
  pl.jobs = (int*)take((size_t)pl.tiles * 4);
  pl.part = (float*)take((size_t)pl.tiles * 2 * pl.dpad * 4);
  return off;
}

template <typename T>
static int launch_embed_bwd(const T* dout, long long ld, const int* tok, int n, int vocab, int d, float scale, int accumulate,
                            float* grad, unsigned* status, void* ws, cudaStream_t s) {
  EmbedPlan pl;
  embed_plan(pl, n, vocab, d, ws);
  int key_bits = 1;
  while ((vocab >> key_bits) != 0) ++key_bits;                     // keys 0 .. vocab
  const int passes = ceil_div(key_bits, 8), bits = ceil_div(key_bits, passes);
  pl.sorted = pl.buf[(passes - 1) & 1];
  const int ranks = n > 8192 ? ES_MAX_RANKS : 1;                   // one block sorts a short batch sooner than eight that exchange counts
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ranks);
  cfg.blockDim = dim3(ES_THREADS);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, embed_sort_kernel, tok, pl, ranks, passes, bits, status) != cudaSuccess) {
    cudaGetLastError();
    return PCM_ERR_CUDA;
  }
  g_launches.fetch_add(1, std::memory_order_relaxed);
  const bool vec = !(((uintptr_t)dout | (uintptr_t)grad) & 15) && d % Vec16<T>::N == 0 && ld % Vec16<T>::N == 0;
  const int steps = vec ? d / Vec16<T>::N : d;
  int lg = 0;
  while (lg < 7 && (1 << lg) < steps) ++lg;
  const int slabs = ceil_div(steps, 1 << lg);
  const long long tile_blocks = (long long)ceil_div(pl.tiles, 128 >> lg) * slabs;
  const long long blocks = tile_blocks + (accumulate ? 0 : ceil_div(vocab, 32));
  if (blocks > 0x7FFFFFFFll) return PCM_ERR_SHAPE;
  if (vec) embed_sum_kernel<T, true><<<(unsigned)blocks, 128, 0, s>>>(dout, ld, pl, scale, grad, accumulate, lg, slabs, (int)tile_blocks);
  else embed_sum_kernel<T, false><<<(unsigned)blocks, 128, 0, s>>>(dout, ld, pl, scale, grad, accumulate, lg, slabs, (int)tile_blocks);
  PCM_LAUNCH_CHECK();
  embed_join_kernel<<<dim3(ceil_div(pl.tiles, 8), ceil_div(d, 128)), 256, 0, s>>>(pl, scale, grad, accumulate);
  PCM_LAUNCH_CHECK();
  return PCM_OK;
}

template <typename T>
static int launch_logp(const LogpParams& p, cudaStream_t s) {
  constexpr int NT = 256;
  if (p.V <= 1024) {
    token_logp_kernel<T, 32><<<(unsigned)ceil_div(p.M, 8), 256, 0, s>>>(p, 1);
    PCM_LAUNCH_CHECK();
    return PCM_OK;
  }
  int ranks = 1;
  while (ranks < LP_MAX_RANKS && (long long)p.M * ranks * 2 <= 4ll * sm_count() && p.V / (ranks * 2) >= 2048) ranks *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.M * ranks));
  cfg.blockDim = dim3(NT);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, token_logp_kernel<T, NT>, p, ranks) != cudaSuccess) {
    cudaGetLastError();
    return PCM_ERR_CUDA;
  }
  g_launches.fetch_add(1, std::memory_order_relaxed);
  return PCM_OK;
}

template <typename T>
static int launch_logp_bwd(const LogpBwdParams& p, cudaStream_t s) {
  // 16-byte accesses need every row of logits and gradient to start at the same offset from a 16-byte boundary
  const long long off = (long long)((uintptr_t)p.logits & 15) - (long long)((uintptr_t)p.dlogits & 15);
  const bool vec = off == 0 && ((p.ld - p.ld_d) * (long long)sizeof(T)) % 16 == 0;
  const int per = vec ? LB_THREADS * 2 * Vec16<T>::N : LB_THREADS * 8;
  const int chunks = ceil_div(p.V, per);
  const long long blocks = (long long)p.M * chunks;
  if (blocks > 0x7FFFFFFFll) return PCM_ERR_SHAPE;
  if (vec) token_logp_bwd_kernel<T, true><<<(unsigned)blocks, LB_THREADS, 0, s>>>(p, chunks);
  else token_logp_bwd_kernel<T, false><<<(unsigned)blocks, LB_THREADS, 0, s>>>(p, chunks);
  PCM_LAUNCH_CHECK();
  return PCM_OK;
}

static bool dtype_ok(int32_t dtype) { return dtype == GRPO_F32 || dtype == GRPO_BF16; }
static bool elem_aligned(const void* q, int32_t dtype) { return !((uintptr_t)q & (dtype == GRPO_BF16 ? 1 : 3)); }

}  // namespace pcm

using namespace pcm;

extern "C" int grpo_embed(int32_t dtype, const void* table, int64_t ld_table, int32_t vocab, int32_t d, const int32_t* tok,
                          int32_t n, float scale, void* out, int64_t ld_out, uint32_t* device_status, pcm_stream stream) {
  if (!dtype_ok(dtype) || n < 0 || vocab < 1 || d < 1 || ld_table < d || ld_out < d || !std::isfinite(scale)) return PCM_ERR_ARG;
  if (n == 0) return PCM_OK;
  if (!table || !tok || !out || !elem_aligned(table, dtype) || !elem_aligned(out, dtype)) return PCM_ERR_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  const double es = dtype == GRPO_BF16 ? 2.0 : 4.0;
  prof_begin(PC_EMBED, s);
  const int rc = dtype == GRPO_BF16
                     ? launch_embed((const __nv_bfloat16*)table, ld_table, vocab, d, tok, n, scale, (__nv_bfloat16*)out, ld_out, device_status, s)
                     : launch_embed((const float*)table, ld_table, vocab, d, tok, n, scale, (float*)out, ld_out, device_status, s);
  prof_end(s, (double)n * d, 2.0 * n * d * es);
  return rc;
}

extern "C" size_t grpo_embed_workspace_bytes(int32_t n, int32_t vocab, int32_t d) {
  if (n < 0 || vocab < 1 || d < 1 || d > PCM_MAX_EMBED_DIM) return 0;
  EmbedPlan pl;
  return embed_plan(pl, n, vocab, d, nullptr) + 256;
}

extern "C" int grpo_embed_bwd(int32_t dtype, const void* dout, int64_t ld_dout, const int32_t* tok, int32_t n, int32_t vocab,
                              int32_t d, float scale, uint32_t flags, float* grad, uint32_t* device_status, void* workspace,
                              size_t workspace_bytes, pcm_stream stream) {
  if (!dtype_ok(dtype) || n < 0 || vocab < 1 || d < 1 || ld_dout < d || !std::isfinite(scale) || !grad) return PCM_ERR_ARG;
  if (((uintptr_t)grad & 3) || (flags & ~GRPO_ACCUMULATE)) return PCM_ERR_ARG;
  if (d > PCM_MAX_EMBED_DIM) return PCM_ERR_SHAPE;
  cudaStream_t s = (cudaStream_t)stream;
  const bool accumulate = flags & GRPO_ACCUMULATE;
  if (n == 0) {
    if (!accumulate) PCM_CUDA_TRY(cudaMemsetAsync(grad, 0, (size_t)vocab * d * sizeof(float), s));
    return PCM_OK;
  }
  if (!dout || !tok || !elem_aligned(dout, dtype)) return PCM_ERR_ARG;
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < grpo_embed_workspace_bytes(n, vocab, d)) return PCM_ERR_WORKSPACE;
  prof_begin(PC_EMBED, s);
  const int rc = dtype == GRPO_BF16
                     ? launch_embed_bwd((const __nv_bfloat16*)dout, ld_dout, tok, n, vocab, d, scale, accumulate, grad, device_status, workspace, s)
                     : launch_embed_bwd((const float*)dout, ld_dout, tok, n, vocab, d, scale, accumulate, grad, device_status, workspace, s);
  prof_end(s, 2.0 * n * d, (double)n * d * (dtype == GRPO_BF16 ? 2.0 : 4.0) + 4.0 * vocab * d);
  return rc;
}

extern "C" int grpo_token_logp(int32_t dtype, const void* logits, int64_t ld, int32_t n_rows, int32_t vocab, const int32_t* tok,
                               float temperature, int32_t top, float* logp, float* entropy, float* lse, int32_t* top_id,
                               float* top_logp, uint32_t* device_status, pcm_stream stream) {
  if (!dtype_ok(dtype) || n_rows < 0 || vocab < 1 || ld < vocab || top < 0) return PCM_ERR_ARG;
  if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.f / temperature)) return PCM_ERR_ARG;
  if (top > PCM_MAX_TOP || top > vocab) return PCM_ERR_SHAPE;
  if (n_rows == 0) return PCM_OK;
  if (!logits || !elem_aligned(logits, dtype) || (logp && !tok) || (top > 0 && (!top_id || !top_logp))) return PCM_ERR_ARG;
  const LogpParams p{logits, ld, n_rows, vocab, tok, 1.f / temperature, top, logp, entropy, lse, top_id, top_logp, device_status};
  cudaStream_t s = (cudaStream_t)stream;
  prof_begin(PC_LOSS, s);
  const int rc = dtype == GRPO_BF16 ? launch_logp<__nv_bfloat16>(p, s) : launch_logp<float>(p, s);
  prof_end(s, 5.0 * n_rows * vocab, (double)n_rows * vocab * (dtype == GRPO_BF16 ? 2.0 : 4.0));
  return rc;
}

extern "C" int grpo_token_logp_bwd(int32_t dtype, const void* logits, int64_t ld, int32_t n_rows, int32_t vocab,
                                   const int32_t* tok, float temperature, const float* lse, const float* entropy,
                                   const float* dlogp, const float* dentropy, void* dlogits, int64_t ld_dlogits,
                                   uint32_t* device_status, pcm_stream stream) {
  if (!dtype_ok(dtype) || n_rows < 0 || vocab < 1 || ld < vocab || ld_dlogits < vocab) return PCM_ERR_ARG;
  if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.f / temperature)) return PCM_ERR_ARG;
  if (n_rows == 0) return PCM_OK;
  if (!logits || !tok || !lse || !dlogp || !dlogits || (dentropy && !entropy)) return PCM_ERR_ARG;
  if (!elem_aligned(logits, dtype) || !elem_aligned(dlogits, dtype)) return PCM_ERR_ARG;
  if (dlogits == logits && ld != ld_dlogits) return PCM_ERR_ARG;
  const LogpBwdParams p{logits, ld, dlogits, ld_dlogits, n_rows, vocab, tok, lse, entropy, dlogp, dentropy, 1.f / temperature,
                        device_status};
  cudaStream_t s = (cudaStream_t)stream;
  prof_begin(PC_LOSS, s);
  const int rc = dtype == GRPO_BF16 ? launch_logp_bwd<__nv_bfloat16>(p, s) : launch_logp_bwd<float>(p, s);
  prof_end(s, 7.0 * n_rows * vocab, 2.0 * n_rows * vocab * (dtype == GRPO_BF16 ? 2.0 : 4.0));
  return rc;
}
