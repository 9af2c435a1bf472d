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
// Embedding lookup: out[i] = round(scale * table[tok[i]]); rows of a token outside [0, vocab) are zero.  COPY (scale 1) moves
// bits: a NaN keeps its payload, which a product and a conversion would change.
// Bound by HBM (each distinct row read once, every output row written once); a block holds 256 / tpr rows, tpr
// threads walk one row in 16-byte steps, four loads in flight each.  119808 rows of 1024 bf16 from 32000: 46 - 48 us, 6.5 - 6.7
// TB/s; 64 rows of 2048: 1.5 us.
// ------------------------------------------------------------------------------------------------
template <typename T, bool VEC, bool COPY>
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
        if constexpr (COPY) {                 // rows without a token were read as zeros
          if (v < nv) __stcs(d4 + v, r[u]);
        } else {
          float f[V::N];
          V::unpack(r[u], f);
#pragma unroll
          for (int e = 0; e < V::N; ++e) f[e] *= scale;
          if (v < nv) __stcs(d4 + v, live ? V::pack(f) : make_uint4(0, 0, 0, 0));
        }
      }
    }
  } else {
    for (int c = lane; c < d; c += tpr) dst[c] = !live ? from_f32<T>(0.f) : COPY ? src[c] : from_f32<T>(as_f32(src[c]) * scale);
  }
}

// ------------------------------------------------------------------------------------------------
// Gradient of the embedding: grad[v] (+)= scale * sum over {i : tok[i] = v} of dout[i], in fp32 and in a fixed order.
//   1. (token, position) pairs into token order, stably: few by a bitonic network in one block, more by a radix sort of
//      8-bit digits over up to 256 blocks;
//   2. embed_sum_kernel: tiles of `rows` sorted pairs, each summed in order; a token that crosses more than one border
//      between tiles leaves a partial sum per tile;
//   3. embed_join_kernel: the partial sums of those tokens, in an order that depends on the token's tiles alone.
// Every sum has a fixed order: the same inputs give the same bits.  Bound by HBM: dout once, grad once.  119808 rows of 1024
// bf16 into 32000: 98 - 100 us against 58 us for the bytes; about 18 us are the four sort kernels, which are latency, 57 us the
// sums (5.6 TB/s) and the rest the joins and the rows of absent tokens.
// ------------------------------------------------------------------------------------------------
constexpr int EJ_WARPS = 16, EM_RING = 8, EM_LANES = 16;
constexpr int ES_THREADS = 1024, ES_WARPS = ES_THREADS / 32, ES_BINS = 256, ES_MAX_BLOCKS = 256, ES_SMALL = 2048;

struct EmbedPlan {
  int n, vocab, d;
  int rows, tiles, dpad;                      // sorted pairs per tile, tiles, floats per partial row
  int keys, blocks;                           // pairs per block of the radix sort (a multiple of 1024), blocks
  uint2* buf[2];                              // (token, position) pairs
  unsigned* hist;                             // [blocks][256] digit counts of a block's pairs
  uint8_t* present;                           // [vocab] 1 where a token occurs: marked by its sums, so once for each tile
  int* n_jobs; uint2* jobs;                   // (token, last tile) of every token that left parts
  int* first_tile;                            // [vocab] for those tokens: the tile that they begin in
  float* part;                                // [tiles][2][dpad]: of a token that began before the tile, of one that goes on behind it
  const uint2* sorted;                        // the buffer that the sort ends in
};

// Tokens outside the vocabulary take the key behind its last one.
__device__ __forceinline__ unsigned embed_key(int t, int vocab) { return t >= 0 && t < vocab ? (unsigned)t : (unsigned)vocab; }

// Few pairs: a bitonic network over keys (token above, position below: positions differ, so the order is the stable one)
// in one block, E neighbouring keys a thread.  Exchanges inside a thread need nothing, those inside a warp are shuffles,
// the others go through shared memory.
template <typename K, int POS_BITS, int E>
__global__ void __launch_bounds__(ES_SMALL / E)
embed_sort_small_kernel(const int* __restrict__ tok, const EmbedPlan pl, unsigned* status) {
  __shared__ K sm[2][ES_SMALL];
  const int t = threadIdx.x, T = blockDim.x, base = t * E;
  K key[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = base + e;
    key[e] = ~(K)0;
    if (i < pl.n) {
      const int v = tok[i];
      if (v >= pl.vocab && status) atomicOr(status, STATUS_BAD_TOKEN);
      key[e] = ((K)embed_key(v, pl.vocab) << POS_BITS) | (K)i;
    }
  }
  for (int v = t; v < (pl.vocab + 15) / 16; v += T) reinterpret_cast<uint4*>(pl.present)[v] = make_uint4(0, 0, 0, 0);
  if (t == 0) *pl.n_jobs = 0;
  int turn = 0;
  for (int k = 2; k <= T * E; k <<= 1) {
    for (int j = k >> 1; j >= E; j >>= 1) {   // partner in another thread
      const bool lower = (base & j) == 0, up = (base & k) == 0;       // the same for the thread's keys: j, k >= E
      const int far = j / E;
      if (far >= 32) {                        // two buffers in turn: one barrier an exchange
#pragma unroll
        for (int e = 0; e < E; ++e) sm[turn][e * T + t] = key[e];
        __syncthreads();
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const K other = far >= 32 ? sm[turn][e * T + (t ^ far)] : __shfl_xor_sync(0xffffffffu, key[e], far & 31);
        const K lo = key[e] < other ? key[e] : other, hi = key[e] < other ? other : key[e];
        key[e] = lower == up ? lo : hi;
      }
      if (far >= 32) turn ^= 1;
    }
#pragma unroll
    for (int j = E / 2; j >= 1; j >>= 1) {    // partner in the same thread
      if (j > k >> 1) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (e & j) continue;
        const bool up = ((base + e) & k) == 0;
        const K a = key[e], b = key[e | j], lo = a < b ? a : b, hi = a < b ? b : a;
        key[e] = up ? lo : hi;
        key[e | j] = up ? hi : lo;
      }
    }
  }
  let_successor_start();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (base + e < pl.n) pl.buf[0][base + e] = make_uint2((unsigned)(key[e] >> POS_BITS), (unsigned)key[e] & ((1u << (POS_BITS < 32 ? POS_BITS : 31)) - 1u));
}

// Digit counts of one pass for each block's pairs.  The first one also clears what the sums will mark.
__global__ void __launch_bounds__(ES_THREADS)
embed_count_kernel(const int* __restrict__ tok, const EmbedPlan pl, int pass, int bits, unsigned* status) {
  __shared__ unsigned count[ES_BINS];
  const int tid = threadIdx.x;
  if (tid < ES_BINS) count[tid] = 0;
  __syncthreads();
  const unsigned mask = (1u << bits) - 1u;
  const long long lo = (long long)blockIdx.x * pl.keys, hi = min(lo + pl.keys, (long long)pl.n);
  if (pass == 0) {
    const long long first = (long long)blockIdx.x * ES_THREADS + tid, stride = (long long)gridDim.x * ES_THREADS;
    for (long long v = first; v < (pl.vocab + 15) / 16; v += stride) reinterpret_cast<uint4*>(pl.present)[v] = make_uint4(0, 0, 0, 0);
    if (first == 0) *pl.n_jobs = 0;
    let_successor_start();
    for (long long i = lo + tid; i < hi; i += ES_THREADS) {
      const int t = tok[i];
      if (t >= pl.vocab && status) atomicOr(status, STATUS_BAD_TOKEN);
      atomicAdd(&count[embed_key(t, pl.vocab) & mask], 1u);
    }
  } else {
    wait_for_predecessor();
    let_successor_start();
    const uint2* src = (pass & 1) ? pl.buf[0] : pl.buf[1];
    for (long long i = lo + tid; i < hi; i += ES_THREADS) atomicAdd(&count[(__ldcg(src + i).x >> (pass * bits)) & mask], 1u);
  }
  __syncthreads();
  if (tid < ES_BINS) pl.hist[blockIdx.x * ES_BINS + tid] = count[tid];
}

// Lanes of the warp that hold the same digit as this one, among the lanes with `in`: a ballot for each bit of the digit.
__device__ __forceinline__ unsigned same_digit(unsigned dig, bool in, int bits) {
  unsigned same = __ballot_sync(0xffffffffu, in);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    if (b < bits) {
      const bool on = (dig >> b) & 1u;
      const unsigned ones = __ballot_sync(0xffffffffu, on);
      same &= on ? ones : ~ones;
    }
  }
  return same;
}

// One pass: every pair to where its digit puts it, 1024 pairs of the block at a time in their order.  (Counting the next
// pass's digits here, by atomics on the blocks that the pairs land in, took 8 us of 119808 pairs; its own kernel takes 4.)
__global__ void __launch_bounds__(ES_THREADS)
embed_scatter_kernel(const int* __restrict__ tok, const EmbedPlan pl, int pass, int bits) {
  __shared__ unsigned count[ES_WARPS][ES_BINS];
  __shared__ unsigned sums[2][ES_WARPS * 32 / ES_BINS][ES_BINS];
  __shared__ unsigned base[ES_BINS], warp_sum[ES_BINS / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long lo = (long long)blockIdx.x * pl.keys, hi = min(lo + pl.keys, (long long)pl.n);
  const int first_tok = pass == 0 && lo + tid < hi ? tok[lo + tid] : 0;      // an input: it need not wait
  wait_for_predecessor();
  const unsigned* hist = pl.hist;
  const uint2* src = (pass & 1) ? pl.buf[0] : pl.buf[1];
  uint2* dst = (pass & 1) ? pl.buf[1] : pl.buf[0];
  const unsigned mask = (1u << bits) - 1u;
  const int shift = pass * bits;
  {
    // per digit: pairs in all blocks and in the blocks before this one; four threads share a digit
    const int dig = tid & (ES_BINS - 1), q = tid / ES_BINS, quarter = ES_THREADS / ES_BINS;
    unsigned before = 0, all = 0;
#pragma unroll 8
    for (int b = q; b < pl.blocks; b += quarter) {
      const unsigned k = __ldcg(hist + b * ES_BINS + dig);
      all += k;
      before += b < (int)blockIdx.x ? k : 0;
    }
    sums[0][q][dig] = all;
    sums[1][q][dig] = before;
  }
  __syncthreads();
  if (tid < ES_BINS) {
    unsigned all = 0, before = 0;
    for (int q = 0; q < ES_THREADS / ES_BINS; ++q) { all += sums[0][q][tid]; before += sums[1][q][tid]; }
    unsigned incl = all;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const unsigned o = __shfl_up_sync(0xffffffffu, incl, off);
      incl += lane >= off ? o : 0;
    }
    if (lane == 31) warp_sum[warp] = incl;
    base[tid] = incl - all + before;
  }
  __syncthreads();
  if (tid < ES_BINS)
    for (int w = 0; w < warp; ++w) base[tid] += warp_sum[w];
  let_successor_start();
  for (long long i0 = lo; i0 < hi; i0 += ES_THREADS) {
    const long long i = i0 + tid;
    const bool in = i < hi;
    uint2 kv = make_uint2(0u, 0u);
    if (in) kv = pass == 0 ? make_uint2(embed_key(i0 == lo ? first_tok : tok[i], pl.vocab), (unsigned)i) : __ldcg(src + i);
    for (int k = tid; k < ES_WARPS * ES_BINS; k += ES_THREADS) (&count[0][0])[k] = 0;
    __syncthreads();
    const unsigned dig = (kv.x >> shift) & mask;
    const unsigned same = same_digit(dig, in, bits);
    if (in && lane == __ffs(same) - 1) count[warp][dig] = __popc(same);
    __syncthreads();
    unsigned total = 0;
    if (tid < ES_BINS) {                      // per digit: the warps' counts into where each warp's pairs begin
#pragma unroll 8
      for (int w = 0; w < ES_WARPS; ++w) {
        const unsigned k = count[w][tid];
        count[w][tid] = total;
        total += k;
      }
    }
    __syncthreads();
    if (in) {
      const unsigned at = base[dig] + count[warp][dig] + __popc(same & ((1u << lane) - 1u));
      dst[at] = kv;
    }
    __syncthreads();
    if (tid < ES_BINS) base[tid] += total;
  }
}

// A warp sums one tile (up to 32 sorted pairs, one per lane) over the columns of its slab: NV pieces of 16 bytes (or of one
// element) per lane.  What a row needs besides its bytes is kept small, because instructions, not bytes,
// bounded the version in which every thread looked at every pair: which rows open a token and which count comes
// from two ballots.
template <typename T, bool VEC>
__global__ void __launch_bounds__(128)
embed_sum_kernel(const T* __restrict__ dout, long long ld, const float* __restrict__ coef, const EmbedPlan pl, float scale,
                 float* __restrict__ grad, int accumulate, int slabs) {
  constexpr int N = VEC ? Vec16<T>::N : 1, NV = VEC ? 2 : 4, U = 8;
  wait_for_predecessor();
  let_successor_start();
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  // Tiles run in EM_LANES interleaved sequences: where tokens are numbered by frequency, one sequence would read (many rows
  // of a token) first and write (a token a row) last (97 us, 111 in one sequence).
  const int place = (int)(item / slabs), slab = (int)(item - (long long)place * slabs);
  const int per = (pl.tiles + EM_LANES - 1) / EM_LANES, tile = (place % EM_LANES) * per + place / EM_LANES;
  if (place / EM_LANES >= per || tile >= pl.tiles) return;
  const uint2* pair = pl.sorted;
  const int lo = tile * pl.rows, hi = min(lo + pl.rows, pl.n);
  const unsigned none = 0xFFFFFFFFu, vocab = (unsigned)pl.vocab;
  auto pair_at = [&](long long i, long long end) { return i < end ? pair[i] : make_uint2(none, 0u); };
  const uint2 own = pair_at(lo + lane, hi);
  const uint2 beyond = pair_at((long long)hi + lane, min((long long)hi + pl.rows, (long long)pl.n));
  // A token that crosses one border between tiles belongs to the tile it begins in; one that crosses more leaves a part
  // in every tile it touches.
  const unsigned head = __shfl_sync(0xffffffffu, own.x, 0), tail = __shfl_sync(0xffffffffu, own.x, hi - lo - 1);
  const unsigned behind = __shfl_sync(0xffffffffu, beyond.x, 0);
  const unsigned before = lo > 0 ? pair[lo - 1].x : none, far_before = lo > pl.rows ? pair[lo - pl.rows - 1].x : none;
  const unsigned far_behind = (long long)hi + pl.rows < pl.n ? pair[hi + pl.rows].x : none;
  const bool head_on = before == head;                                         // began before this tile
  const bool tail_on = behind == tail && !(head_on && head == tail);           // begins here and goes on behind it
  const bool head_far = head_on && (far_before == head || behind == head);
  const bool tail_far = tail_on && far_behind == tail;
  const unsigned skip = head_on && !head_far ? head : none;                    // the tile before sums it
  int col[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) col[j] = (slab * NV + j) * 32 * N + lane * N;
  unsigned cur = none;
  float acc[NV][N];
  // Added by the memory, not read back: an element has one addition per call, so there is no order to depend on, and a
  // warp does not wait for the row it adds to.
  auto put = [&](float* dst, const float (&a)[N], float f, bool add) {
    if constexpr (N >= 4) {
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        if (add) red_add_v4(dst + e, a[e] * f, a[e + 1] * f, a[e + 2] * f, a[e + 3] * f);
        else *reinterpret_cast<float4*>(dst + e) = make_float4(a[e] * f, a[e + 1] * f, a[e + 2] * f, a[e + 3] * f);
      }
    } else if (add) {
      atomicAdd(dst, a[0] * f);
    } else {
      dst[0] = a[0] * f;
    }
  };
  auto flush = [&]() {
    if (cur == none) return;
    if (slab == 0 && lane == 0) pl.present[cur] = 1;
    float* dst = grad + (long long)cur * pl.d;
    float f = scale;
    bool add = accumulate != 0;
    if (head_far && cur == head) {
      dst = pl.part + ((long long)tile * 2) * pl.dpad;
      f = 1.f; add = false;
      if (slab == 0 && lane == 0 && behind != head) pl.jobs[atomicAdd(pl.n_jobs, 1)] = make_uint2(head, (unsigned)tile);    // it ends here
    } else if (tail_far && cur == tail) {
      dst = pl.part + ((long long)tile * 2 + 1) * pl.dpad;
      f = 1.f; add = false;
      if (slab == 0 && lane == 0) pl.first_tile[tail] = tile;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (col[j] < pl.d) put(dst + col[j], acc[j], f, add);
  };
  // `kv`: up to 32 pairs, one per lane; rows with a bit in `live` count, those with one in `open` begin a token
  auto begin = [&](unsigned key) {
    flush();
    cur = key;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) acc[j][e] = 0.f;
  };
  auto run = [&](const uint2& kv, unsigned live, unsigned open) {
    const int rows = 32 - __clz(live), first = live ? __ffs(live) - 1 : 0;
    const float weight = coef && ((live >> lane) & 1u) ? coef[kv.y] : 1.f;     // of this lane's row
    if constexpr (VEC) {
      // Every lane copies its own 16-byte pieces of a row into its own shared memory, EM_RING - 1 rows ahead of the sums:
      // bytes in flight without registers, and nobody to wait for but itself.
      extern __shared__ uint4 ring[];         // [4 warps][EM_RING][NV][32]
      uint4* mine = ring + (threadIdx.x >> 5) * (EM_RING * NV * 32) + lane;
      auto issue = [&](int i) {
        const unsigned at = __shfl_sync(0xffffffffu, kv.y, i & 31);
        if (i < rows && ((live >> i) & 1u)) {
          const T* q = dout + (long long)at * ld;
#pragma unroll
          for (int j = 0; j < NV; ++j)
            if (col[j] < pl.d)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(mine + ((i & (EM_RING - 1)) * NV + j) * 32)), "l"(q + col[j])
                           : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
      __syncwarp();
#pragma unroll
      for (int i = 0; i < EM_RING - 1; ++i) issue(first + i);
      for (int i = first; i < rows; ++i) {
        __syncwarp();                         // the row before has been read: its place may be filled again
        issue(i + EM_RING - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(EM_RING - 1) : "memory");
        if (!((live >> i) & 1u)) continue;
        if ((open >> i) & 1u) begin(__shfl_sync(0xffffffffu, kv.x, i));
        const float k = __shfl_sync(0xffffffffu, weight, i);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          float f[N];
          Vec16<T>::unpack(mine[((i & (EM_RING - 1)) * NV + j) * 32], f);
#pragma unroll
          for (int e = 0; e < N; ++e) acc[j][e] += k * f[e];
        }
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    } else {
      for (int i0 = first & ~(U - 1); i0 < rows; i0 += U) {
        float one[U][NV];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const unsigned at = __shfl_sync(0xffffffffu, kv.y, i0 + u);
          if ((live >> (i0 + u)) & 1u) {
            const T* q = dout + (long long)at * ld;
#pragma unroll
            for (int j = 0; j < NV; ++j) one[u][j] = col[j] < pl.d ? as_f32(q[col[j]]) : 0.f;
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (!((live >> (i0 + u)) & 1u)) continue;
          if ((open >> (i0 + u)) & 1u) begin(__shfl_sync(0xffffffffu, kv.x, i0 + u));
          const float k = __shfl_sync(0xffffffffu, weight, i0 + u);
#pragma unroll
          for (int j = 0; j < NV; ++j) acc[j][0] += k * one[u][j];
        }
      }
    }
  };
  const unsigned prev = __shfl_up_sync(0xffffffffu, own.x, 1);
  run(own, __ballot_sync(0xffffffffu, own.x < vocab && own.x != skip), __ballot_sync(0xffffffffu, lane == 0 || prev != own.x));
  if (tail_on && !tail_far) run(beyond, __ballot_sync(0xffffffffu, beyond.x == tail && tail < vocab), 0u);
  flush();
}

// Zeros into the rows of the tokens from v0 on, EJ_WARPS of them, that do not occur.
__device__ void zero_absent_rows(const EmbedPlan& pl, float* __restrict__ grad, long long v0) {
  const long long v = v0 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (v >= pl.vocab || pl.present[v]) return;
  float* g = grad + v * pl.d;
  if (!((uintptr_t)grad & 15) && pl.d % 4 == 0) {
    for (int c = lane * 4; c < pl.d; c += 128) __stcs(reinterpret_cast<float4*>(g + c), make_float4(0.f, 0.f, 0.f, 0.f));
  } else {
    for (int c = lane; c < pl.d; c += 32) g[c] = 0.f;
  }
}

// The first blocks: one warp per token that left parts and 32 columns, its tiles in four slices (eight lanes each, four
// columns a lane); a token over more than 64 tiles is shared by the block's warps.  The slices depend on the token's tiles
// alone.  The other blocks write the rows of absent tokens: stores that need HBM and little else, next to sums that wait
// for one load after the other.
__global__ void __launch_bounds__(EJ_WARPS * 32)
embed_join_kernel(const EmbedPlan pl, float scale, float* __restrict__ grad, int accumulate, int groups, int slabs) {
  __shared__ float4 sum[EJ_WARPS][8];
  __shared__ unsigned key[EJ_WARPS];
  __shared__ int first[EJ_WARPS], span[EJ_WARPS];           // tiles: the first one, how many
  constexpr int LONG = 64;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, slice = lane >> 3;
  wait_for_predecessor();
  if ((int)blockIdx.x >= groups * slabs) {
    zero_absent_rows(pl, grad, (long long)(blockIdx.x - groups * slabs) * EJ_WARPS);
    return;
  }
  const int n_jobs = *pl.n_jobs;
  const int group = blockIdx.x / slabs, col = ((blockIdx.x - group * slabs) * 8 + (lane & 7)) * 4;
  const bool in = col < pl.d;                 // partial rows are padded to a multiple of four
  // partial sums of tiles t + lo .. t + hi - 1 (0: the first tile), then of the warp's four slices
  auto add_tiles = [&](int t, int lo, int hi) {
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    if (in) {
#pragma unroll 8
      for (int k = lo; k < hi; ++k) {
        const float* q = pl.part + ((long long)(t + k) * 2 + (k == 0 ? 1 : 0)) * pl.dpad + col;
        const float4 w = *reinterpret_cast<const float4*>(q);
        a.x += w.x; a.y += w.y; a.z += w.z; a.w += w.w;
      }
    }
#pragma unroll
    for (int off = 8; off < 32; off <<= 1) {
      a.x += __shfl_xor_sync(0xffffffffu, a.x, off);
      a.y += __shfl_xor_sync(0xffffffffu, a.y, off);
      a.z += __shfl_xor_sync(0xffffffffu, a.z, off);
      a.w += __shfl_xor_sync(0xffffffffu, a.w, off);
    }
    return a;
  };
  auto finish = [&](const float4& a, unsigned token) {
    if (!in || slice != 0) return;
    float* g = grad + (long long)token * pl.d + col;
    const float v[4] = {a.x * scale, a.y * scale, a.z * scale, a.w * scale};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < pl.d) g[e] = accumulate ? g[e] + v[e] : v[e];
  };
  // Warp w takes the job `groups * w` behind its block's first: frequent tokens mostly have neighbouring numbers, and so
  // neighbouring jobs, which then fall to different blocks.
  for (int base = group; base < n_jobs; base += groups * EJ_WARPS) {
    const int at = base + warp * groups;
    if (at < n_jobs) {
      const uint2 job = pl.jobs[at];
      const int t = pl.first_tile[job.x], len = (int)job.y - t + 1;
      if (lane == 0) { key[warp] = job.x; first[warp] = t; span[warp] = len; }
      if (len <= LONG) finish(add_tiles(t, len * slice / 4, len * (slice + 1) / 4), job.x);
    } else if (lane == 0) {
      span[warp] = 0;
    }
    __syncthreads();
    for (int j = 0; j < EJ_WARPS; ++j) {
      const int len = span[j];
      if (len <= LONG) continue;              // the same for the whole block
      const int piece = warp * 4 + slice;
      float4 a = add_tiles(first[j], (int)((long long)len * piece / (4 * EJ_WARPS)), (int)((long long)len * (piece + 1) / (4 * EJ_WARPS)));
      if (slice == 0) sum[warp][lane] = a;
      __syncthreads();
      if (warp == 0) {
        a = sum[0][lane & 7];
        for (int w = 1; w < EJ_WARPS; ++w) {
          const float4 b = sum[w][lane & 7];
          a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
        }
        finish(a, key[j]);
      }
      __syncthreads();
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

// Largest element of four 16-byte vectors, NaN if one is.
template <typename T> __device__ __forceinline__ float batch_max(const uint4 (&r)[4]);
template <> __device__ __forceinline__ float batch_max<float>(const uint4 (&r)[4]) {
  float m = __uint_as_float(r[0].x);
#pragma unroll
  for (int u = 0; u < 4; ++u)
    m = max_nan(max_nan(m, max_nan(__uint_as_float(r[u].x), __uint_as_float(r[u].y))), max_nan(__uint_as_float(r[u].z), __uint_as_float(r[u].w)));
  return m;
}
__device__ __forceinline__ uint32_t max2_bf16(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <> __device__ __forceinline__ float batch_max<__nv_bfloat16>(const uint4 (&r)[4]) {
  uint32_t w = r[0].x;
#pragma unroll
  for (int u = 0; u < 4; ++u) w = max2_bf16(max2_bf16(w, max2_bf16(r[u].x, r[u].y)), max2_bf16(r[u].z, r[u].w));
  return max_nan(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <typename T> __device__ __forceinline__ uint4 vec_of_minus_inf();
template <> __device__ __forceinline__ uint4 vec_of_minus_inf<float>() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
template <> __device__ __forceinline__ uint4 vec_of_minus_inf<__nv_bfloat16>() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }

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

// One pass over the logits, bound by HBM on many rows and next by the exponentials (one per element: 0.7 of the unit's rate
// at 6 TB/s of bf16), by latency on few.  21504 rows of 32000 bf16, calls back to back on the same logits: 213 us without a top
// list (6.5 TB/s), 257 us with the top 4, 315 us with 16; on logits that change from call to call 286 us with the top 4.  8 rows
// of 130011 with the top 8: 9.1 us.
// NT threads work on one row's share.  NT = 32: a warp per row, several rows per block.  Otherwise one block per share,
// `ranks` blocks of a cluster per row.
template <int NT> struct LogpSmem {
  static constexpr int CAP = NT == 32 ? 128 : 256;
  static constexpr int W = NT / 32;
  unsigned long long cand[CAP];               // candidates of the top list: order_of(z) above, ~index below
  unsigned long long warp_best[W];
  unsigned group_max[32];
  VocabStat part[W];
  int warp_count[W];
  int n_cand;
  unsigned long long best[NT == 32 ? 1 : LP_MAX_RANKS * LP_MAX_TOP];   // rank 0: the shares' own top lists
  VocabStat share[NT == 32 ? 1 : LP_MAX_RANKS];
};

template <int NT> __device__ __forceinline__ void row_sync() {
  if constexpr (NT == 32) __syncwarp(); else __syncthreads();
}

__device__ __forceinline__ unsigned long long top_key(float z, int idx) {
  return ((unsigned long long)order_of(z) << 32) | (0xFFFFFFFFu - (unsigned)idx);
}

// The `top` largest elements of a share into sm.cand[0 .. returned), unordered (all of them when the share has fewer).
//   1. The threads form 32 groups; the top-th largest of the groups' maxima, `limit`, is a value that at least `top`
//      elements reach.  Few threads have a maximum that reaches it: their elements are read again, a warp at a time, and
//      those that do go on the list.
//   2. If they do not fit (many equal values: a constant row, a mask that leaves fewer than `top`) or there is a NaN, the
//      list takes what lies above the limit, and then elements equal to it, in ascending order, until it has `top`.
//   3. If not even those fit, one search of the share for each place.
template <int NT>
__device__ __forceinline__ unsigned top_limit(LogpSmem<NT>& sm, int lane, int top) {
  unsigned mine = sm.group_max[lane], limit = 0;
  for (int k = 0; k < top; ++k) {
    limit = __reduce_max_sync(0xffffffffu, mine);
    if (lane == __ffs(__ballot_sync(0xffffffffu, mine == limit)) - 1) mine = 0;
  }
  return limit;
}

template <typename T, int NT>
__device__ __noinline__ int top_list_slow(LogpSmem<NT>& sm, const RowShare<T>& sh, float own, int tid, int top, unsigned limit) {
  using V16 = Vec16<T>;
  constexpr int N = V16::N, W = NT / 32, CAP = LogpSmem<NT>::CAP;
  const int lane = tid & 31, warp = tid >> 5;
  const unsigned own_max = order_of(own);
  row_sync<NT>();
  if (tid == 0) sm.n_cand = 0;
  row_sync<NT>();
  int n = 0;
  if (limit != 0xFFFFFFFFu) {                 // elements above the limit; nothing is above a NaN
    auto offer = [&](float z, int idx) {
      if (order_of(z) > limit) {
        const int at = atomicAdd(&sm.n_cand, 1);
        if (at < CAP) sm.cand[at] = top_key(z, idx);
      }
    };
    for (unsigned owners = __ballot_sync(0xffffffffu, own_max > limit); owners; owners &= owners - 1) {
      if (*reinterpret_cast<volatile int*>(&sm.n_cand) > CAP) break;       // it has overflowed: the rest would be thrown away
      const int owner = warp * 32 + __ffs(owners) - 1;
      for (int v = sh.v_lo + owner + lane * NT; v < sh.v_hi; v += 32 * NT) {
        float f[N];
        V16::unpack(__ldg(sh.vec(v)), f);
#pragma unroll
        for (int k = 0; k < N; ++k) offer(f[k], sh.head + v * N + k);
      }
    }
    const int e = sh.single(tid);
    if (e >= 0) offer(as_f32(sh.p[e]), e);
    row_sync<NT>();
    n = sm.n_cand;
  }
  if (n <= CAP) {
    if (n >= top) return n;
    const int above = n;
    int found = 0;
    // `bits`: which of `count` consecutive elements from `idx` on equal the limit; threads hold them in ascending order
    auto take = [&](unsigned bits, int idx) {
      const int own_n = __popc(bits);
      int incl = own_n;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, off);
        incl += lane >= off ? o : 0;
      }
      int before = found + incl - own_n, total = __shfl_sync(0xffffffffu, incl, 31);
      if constexpr (W > 1) {
        if (lane == 31) sm.warp_count[warp] = incl;
        __syncthreads();
        total = 0;
        for (int w = 0; w < W; ++w) {
          before += w < warp ? sm.warp_count[w] : 0;
          total += sm.warp_count[w];
        }
        __syncthreads();
      }
      for (; bits && above + before < top; bits &= bits - 1, ++before)
        sm.cand[above + before] = ((unsigned long long)limit << 32) | (0xFFFFFFFFu - (unsigned)(idx + __ffs(bits) - 1));
      found += total;
    };
    const int first = tid, last = sh.tail + tid;
    take(sh.has_head && first < sh.head && order_of(as_f32(sh.p[first])) == limit ? 1u : 0u, first);
    for (int v0 = sh.v_lo; v0 < sh.v_hi && above + found < top; v0 += NT) {
      const int v = v0 + tid;
      unsigned bits = 0;
      if (v < sh.v_hi) {
        float f[N];
        V16::unpack(__ldg(sh.vec(v)), f);
#pragma unroll
        for (int k = 0; k < N; ++k) bits |= order_of(f[k]) == limit ? 1u << k : 0u;
      }
      take(bits, sh.head + v * N);
    }
    if (above + found < top) take(sh.has_tail && last < sh.V && order_of(as_f32(sh.p[last])) == limit ? 1u : 0u, last);
    row_sync<NT>();
    return min(top, above + found);
  }
  unsigned long long below = ~0ull;
  for (int place = 0; place < top; ++place) {
    unsigned long long best = 0;
    auto offer = [&](float z, int idx) {
      const unsigned long long key = top_key(z, idx);
      if (key < below && key > best) best = key;
    };
    const int e = sh.single(tid);
    if (e >= 0) offer(as_f32(sh.p[e]), e);
#pragma unroll 4
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
    if constexpr (W > 1) {
      __syncthreads();
      if (lane == 0) sm.warp_best[warp] = best;
      __syncthreads();
      for (int w = 0; w < W; ++w) best = sm.warp_best[w] > best ? sm.warp_best[w] : best;
    }
    if (tid == 0) sm.cand[place] = best;
    below = best;
  }
  row_sync<NT>();
  return top;                                 // more than CAP elements lie above the limit, so there are `top`
}

template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT == 32 ? 256 : NT)
token_logp_kernel(const LogpParams p, int ranks) {
  using V16 = Vec16<T>;
  constexpr int N = V16::N, U = 4, W = NT / 32;
  constexpr int ROWS = NT == 32 ? 8 : 1;
  __shared__ LogpSmem<NT> smem_all[ROWS];
  LogpSmem<NT>& sm = smem_all[NT == 32 ? threadIdx.x >> 5 : 0];
  const int tid = NT == 32 ? threadIdx.x & 31 : threadIdx.x;
  const int lane = threadIdx.x & 31;
  const int rank = NT == 32 || ranks == 1 ? 0 : (int)cluster_ctarank();
  const float c = p.inv_t * VOCAB_LOG2E;
  const int top = TOP ? p.top : 0;
  const long long row = NT == 32 ? (long long)blockIdx.x * ROWS + (threadIdx.x >> 5) : blockIdx.x / ranks;
  if (row >= p.M) return;                     // whole warps (NT = 32) only: the grid is exact otherwise
  const int t = p.tok ? p.tok[row] : 0;
  const bool bad = p.tok && t >= p.V, skip = p.tok && (t < 0 || bad);
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

  // ---- one pass over the share: U vectors at a time, the next U on their way --------------------------------
  // The exponent is held at -1000 or above, so that -inf (and -inf - -inf, a NaN) adds 0 to both sums.
  float m = -INFINITY;
  unsigned long long s2 = pack2(0.f, 0.f), w2 = s2;
  const unsigned long long c2 = pack2(c, c);
  {
    const int e = sh.single(tid);
    if (e >= 0) {
      m = as_f32(sh.p[e]);
      s2 = pack2(m == -INFINITY ? 0.f : 1.f, 0.f);
    }
  }
  auto use = [&](const uint4 (&r)[U]) {
    const float bm = max_nan(batch_max<T>(r), m);
    if (bm != m) {
      const float d = fmaxf((m - bm) * c, -1000.f), f = ex2(d);
      const unsigned long long f2 = pack2(f, f);
      w2 = mul2(f2, fma2(s2, pack2(d, d), w2));
      s2 = mul2(f2, s2);
      m = bm;
    }
    const unsigned long long neg_m = pack2(-m, -m);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      V16::unpack(r[u], f);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        float t0, t1;
        unpack2(mul2(add2(pack2(f[e], f[e + 1]), neg_m), c2), t0, t1);
        t0 = fmaxf(t0, -1000.f);
        t1 = fmaxf(t1, -1000.f);
        const unsigned long long x2 = pack2(ex2(t0), ex2(t1));
        s2 = add2(s2, x2);
        w2 = fma2(x2, pack2(t0, t1), w2);
      }
    }
  };
  {
    const uint4* q = sh.vec(sh.v_lo + tid);
    const int full = (sh.v_hi - sh.v_lo) / (U * NT);
    auto load = [&](uint4 (&r)[U]) {
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = __ldg(q + u * NT);
      q += U * NT;
    };
    uint4 a[U], b[U];
    if (full > 0) load(a);
    for (int k = 0; k < full; k += 2) {
      if (k + 1 < full) load(b);
      use(a);
      if (k + 1 < full) {
        if (k + 2 < full) load(a);
        use(b);
      }
    }
    const int rest = sh.v_hi - sh.v_lo - full * (U * NT);
    if (rest > 0) {                           // missing vectors read as -inf, which adds nothing
#pragma unroll
      for (int u = 0; u < U; ++u) a[u] = tid + u * NT < rest ? __ldg(q + u * NT) : vec_of_minus_inf<T>();
      use(a);
    }
  }

  // ---- join the threads: lanes against their common maximum, then the warps one after the other --------------
  if constexpr (TOP) {
    unsigned g = order_of(m);                 // -inf where the thread has no element: never above an element's
#pragma unroll
    for (int off = 1; off < W; off <<= 1) g = max(g, __shfl_xor_sync(0xffffffffu, g, off));
    if (tid % W == 0) sm.group_max[tid / W] = g;
  }
  VocabStat st;
  {
    float a, b, wa, wb;
    unpack2(s2, a, b);
    unpack2(w2, wa, wb);
    float s = a + b, w = wa + wb;
    asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(st.m) : "f"(m));
    const float d = m == st.m ? 0.f : fmaxf((m - st.m) * c, -1000.f), f = ex2(d);
    w = f * (w + s * d);
    s *= f;
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, off);
      w += __shfl_xor_sync(0xffffffffu, w, off);
    }
    st.s = s;
    st.w = w;
  }
  if constexpr (W > 1) {
    if (lane == 0) sm.part[tid >> 5] = st;
    __syncthreads();
    st = sm.part[0];
#pragma unroll
    for (int w = 1; w < W; ++w) st = stat_join(st, sm.part[w], c);
  } else {
    __syncwarp();
  }

  int n = 0;
  if constexpr (TOP) {
    const unsigned limit = top_limit<NT>(sm, lane, top);
    bool slow = st.m != st.m;
    if (!slow) {
      const float least = float_of_order(limit);
      auto put = [&](float z, int idx) {
        const int at = atomicAdd(&sm.n_cand, 1);
        if (at < LogpSmem<NT>::CAP) sm.cand[at] = top_key(z, idx);
      };
      unsigned owners = __ballot_sync(0xffffffffu, m >= least);
      // nearly every thread of a warp: a constant or masked share, which would only flood the list
      if (W > 1 && __popc(owners) > 24) {
        if (lane == 0) atomicAdd(&sm.n_cand, LogpSmem<NT>::CAP + 1);
        owners = 0;
      }
      while (owners) {                        // four threads' elements at a time, so that their loads overlap
        if (*reinterpret_cast<volatile int*>(&sm.n_cand) > LogpSmem<NT>::CAP) break;
        int from[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          from[j] = owners ? sh.v_lo + (tid & ~31) + __ffs(owners) - 1 : sh.v_hi;
          owners &= owners - 1;
        }
        for (int off = lane * NT; off < sh.v_hi - sh.v_lo; off += 32 * NT) {
          uint4 r[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) r[j] = from[j] < sh.v_hi - off ? __ldg(sh.vec(from[j] + off)) : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (from[j] >= sh.v_hi - off) continue;
            float f[N];
            V16::unpack(r[j], f);
            unsigned bits = 0;
#pragma unroll
            for (int k = 0; k < N; ++k) bits |= f[k] >= least ? 1u << k : 0u;
            for (; bits; bits &= bits - 1) {  // mostly one lane, once
              const int at = __ffs(bits) - 1;
              float z = f[0];
#pragma unroll
              for (int k = 1; k < N; ++k) z = at == k ? f[k] : z;
              put(z, sh.head + (from[j] + off) * N + at);
            }
          }
        }
      }
      const int e = sh.single(tid);
      if (e >= 0 && as_f32(sh.p[e]) >= least) put(as_f32(sh.p[e]), e);
      row_sync<NT>();
      n = sm.n_cand;
      slow = n > LogpSmem<NT>::CAP;
    }
    if (slow) n = top_list_slow<T, NT>(sm, sh, m, tid, top, limit);
  }
  auto place_of = [&](unsigned long long key) {
    int place = 0;
    for (int j = 0; j < n; ++j) place += sm.cand[j] > key ? 1 : 0;
    return place;
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
    for (int i = tid; i < n; i += NT) {
      const unsigned long long key = sm.cand[i];
      const int place = place_of(key);
      if (place < top) write_top(res, place, key);
    }
    return;
  }
  if constexpr (NT > 32) {
    // ---- join the shares of a cluster on rank 0 ----
    cluster_sync_all();                       // rank 0 runs: its shared memory may be written
    const uint32_t share0 = mapa_shared(smem_u32(&sm.share[rank]), 0);
    if (tid == 0) {
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(share0), "f"(st.m) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(share0 + 4u), "f"(st.s) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(share0 + 8u), "f"(st.w) : "memory");
    }
    if constexpr (TOP) {
      const uint32_t best0 = mapa_shared(smem_u32(&sm.best[rank * LP_MAX_TOP]), 0);
      auto put = [&](int place, unsigned long long key) {
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(best0 + (uint32_t)place * 8u), "l"(key) : "memory");
      };
      if (tid >= n && tid < top) put(tid, 0);             // a share with fewer elements than places
      for (int i = tid; i < n; i += NT) {
        const unsigned long long key = sm.cand[i];
        const int place = place_of(key);
        if (place < top) put(place, key);
      }
    }
    cluster_sync_all();
    if (rank != 0) return;
    st = sm.share[0];
    for (int r = 1; r < ranks; ++r) st = stat_join(st, sm.share[r], c);
    const RowResult res(st, p.inv_t);
    if (tid == 0) write_row(res);
    if (TOP && tid < ranks * LP_MAX_TOP && tid % LP_MAX_TOP < top) {
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
// One read and one write of the logits, bound by HBM; a thread reads what it writes, so dlogits may be the logits
// themselves.
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

constexpr int LB_THREADS = 256, LB_VECS = 4;  // 10752 x 32000 bf16: 254 us with two vectors a thread, 221 with four, in
// calls back to back; 241 where the inputs change from call to call

template <typename T, bool VEC>
__global__ void __launch_bounds__(LB_THREADS)
token_logp_bwd_kernel(const LogpBwdParams p, int chunks) {
  using V16 = Vec16<T>;
  constexpr int N = V16::N, U = VEC ? LB_VECS : 8;
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
  const bool copy = scale == 1.f;
  auto kernel = vec ? (copy ? embed_kernel<T, true, true> : embed_kernel<T, true, false>)
                    : (copy ? embed_kernel<T, false, true> : embed_kernel<T, false, false>);
  kernel<<<(unsigned)blocks, 256, 0, s>>>(table, ld_table, vocab, d, tok, n, scale, out, ld_out, status, lg);
  PCM_LAUNCH_CHECK();
  return PCM_OK;
}

static bool sizes_ok(int64_t rows, int64_t vocab) { return rows <= PCM_MAX_VOCAB_CALL && vocab <= PCM_MAX_VOCAB_CALL; }

// Sorted pairs per tile: fewer for short batches, so that every SM gets some.
constexpr int EM_LONG = 32 * 296;
static int embed_tile_rows(int n) { return n >= EM_LONG ? 32 : 8; }

// Every region is as large as any batch of up to n rows needs it, so that a workspace sized for n holds a shorter batch too
// (the last chunk of rows of grpo_head_logp_bwd): just below EM_LONG there are more tiles than just above it, and a sort
// of 262144 pairs runs in more blocks than one of 262145.
static size_t embed_plan(EmbedPlan& pl, int n, int vocab, int d, void* ws) {
  const int most_tiles = max(ceil_div(n, 32), ceil_div(min(n, EM_LONG - 1), 8));
  const int most_blocks = min(ceil_div(n, ES_THREADS), ES_MAX_BLOCKS);
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
  pl.keys = ceil_div(ceil_div(n, ES_MAX_BLOCKS), ES_THREADS) * ES_THREADS;
  if (pl.keys < ES_THREADS) pl.keys = ES_THREADS;
  pl.blocks = ceil_div(n, pl.keys);
  pl.present = (uint8_t*)take((size_t)vocab);
  pl.hist = (unsigned*)take((size_t)most_blocks * ES_BINS * 4);
  pl.n_jobs = (int*)take(4);
  pl.jobs = (uint2*)take((size_t)most_tiles * 8);
  pl.first_tile = (int*)take((size_t)vocab * 4);
  pl.part = (float*)take((size_t)most_tiles * 2 * pl.dpad * 4);
  return off;
}

static int embed_passes(int vocab) {
  int key_bits = 1;
  while ((vocab >> key_bits) != 0) ++key_bits;                     // keys 0 .. vocab
  return ceil_div(key_bits, 8);
}
// One block: up to 2048 pairs whose key fits 32 bits (token and a position of 11), 1024 of any vocabulary.  The gradient of
// 1500 rows of 520 fp32 takes 17 us with the network and 20 with the radix sort, of 4000 rows 25 and 21.
constexpr int ES_SMALL_VOCAB = (1 << 21) - 2;
static bool embed_sorts_small(int n, int vocab) { return n <= (vocab <= ES_SMALL_VOCAB ? ES_SMALL : ES_SMALL / 2); }
static EmbedPlan embed_sorted_plan(int n, int vocab, int d, void* ws) {
  EmbedPlan pl;
  embed_plan(pl, n, vocab, d, ws);
  pl.sorted = embed_sorts_small(n, vocab) ? pl.buf[0] : pl.buf[(embed_passes(vocab) - 1) & 1];
  return pl;
}

static int launch_embed_sort(const EmbedPlan& pl, const int* tok, unsigned* status, cudaStream_t s) {
  const int n = pl.n, vocab = pl.vocab;
  if (embed_sorts_small(n, vocab)) {
    const bool narrow = vocab <= ES_SMALL_VOCAB;
    int threads = 128;
    while (threads * (narrow ? 4 : 2) < n) threads *= 2;
    if (narrow) embed_sort_small_kernel<unsigned, 11, 4><<<1, threads, 0, s>>>(tok, pl, status);
    else embed_sort_small_kernel<unsigned long long, 32, 2><<<1, threads, 0, s>>>(tok, pl, status);
    PCM_LAUNCH_CHECK();
  } else {
    int key_bits = 1;
    while ((vocab >> key_bits) != 0) ++key_bits;
    const int passes = embed_passes(vocab), bits = ceil_div(key_bits, passes);
    const dim3 grid(pl.blocks), block(ES_THREADS);
    for (int pass = 0; pass < passes; ++pass) {
      int rc = PCM_OK;
      if (pass == 0) {
        embed_count_kernel<<<grid, block, 0, s>>>(tok, pl, pass, bits, status);
        PCM_LAUNCH_CHECK();
      } else {
        rc = launch_after(embed_count_kernel, grid, block, s, tok, pl, pass, bits, status);
      }
      if (rc == PCM_OK) rc = launch_after(embed_scatter_kernel, grid, block, s, tok, pl, pass, bits);
      if (rc != PCM_OK) return rc;
    }
  }
  return PCM_OK;
}

template <typename T>
static int launch_embed_sum(const EmbedPlan& pl, const T* dout, long long ld, const float* coef, float scale, int accumulate, float* grad,
                            cudaStream_t s) {
  const int vocab = pl.vocab, d = pl.d;
  const bool vec = !(((uintptr_t)dout | (uintptr_t)grad) & 15) && d % Vec16<T>::N == 0 && ld % Vec16<T>::N == 0;
  const int slabs = ceil_div(d, vec ? 64 * Vec16<T>::N : 128);
  const long long blocks = ((long long)ceil_div(pl.tiles, EM_LANES) * EM_LANES * slabs + 3) / 4;
  if (blocks > 0x7FFFFFFFll) return PCM_ERR_SHAPE;
  const int rc = launch_after_smem(vec ? embed_sum_kernel<T, true> : embed_sum_kernel<T, false>, dim3((unsigned)blocks), dim3(128),
                                   vec ? 4 * EM_RING * 2 * 32 * 16 : 0, s, dout, ld, coef, pl, scale, grad, accumulate, slabs);
  if (rc != PCM_OK) return rc;
  const int join_slabs = ceil_div(d, 32), most = ceil_div(pl.tiles, EJ_WARPS);
  const int groups = pl.tiles <= 2 ? 0 : most < 16 ? most : 16;    // two tiles: nothing crosses two borders
  const int join_blocks = groups * join_slabs + (accumulate ? 0 : ceil_div(vocab, EJ_WARPS));
  if (join_blocks == 0) return PCM_OK;
  return launch_after(embed_join_kernel, dim3(join_blocks), dim3(EJ_WARPS * 32), s, pl, scale, grad, accumulate, groups, join_slabs);
}

size_t embed_accumulate_bytes(int n, int vocab, int d) {
  EmbedPlan pl;
  return embed_plan(pl, n, vocab, d, nullptr);
}
int embed_accumulate_sort(const int* tok, int n, int vocab, int d, void* scratch, size_t scratch_bytes, cudaStream_t s) {
  if (embed_accumulate_bytes(n, vocab, d) > scratch_bytes) return PCM_ERR_WORKSPACE;
  return launch_embed_sort(embed_sorted_plan(n, vocab, d, scratch), tok, nullptr, s);
}
int embed_accumulate_sum(const void* rows, const float* coef, int n, int vocab, int d, float* grad, void* scratch, cudaStream_t s) {
  return launch_embed_sum(embed_sorted_plan(n, vocab, d, scratch), (const __nv_bfloat16*)rows, d, coef, 1.f, 1, grad, s);
}

template <typename T, int NT>
static int launch_logp_as(const LogpParams& p, int ranks, cudaStream_t s) {
  void (*kernel)(LogpParams, int) = p.top > 0 ? token_logp_kernel<T, NT, true> : token_logp_kernel<T, NT, false>;
  if (ranks == 1) {
    // without the cluster attribute: with it, even at one block a cluster, fewer blocks were resident
    kernel<<<NT == 32 ? ceil_div(p.M, 8) : p.M, NT == 32 ? 256 : NT, 0, s>>>(p, 1);
    PCM_LAUNCH_CHECK();
    return PCM_OK;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.M * ranks));
  cfg.blockDim = dim3(NT);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, p, ranks) != cudaSuccess) {
    cudaGetLastError();
    return PCM_ERR_CUDA;
  }
  g_launches.fetch_add(1, std::memory_order_relaxed);
  return PCM_OK;
}

// Short rows: a warp each.  Enough rows to fill the GPU with blocks of 128: one block each (its fixed costs, reductions
// and the top list, weigh least then: 21504 x 32000 top 4 took 279 us, 307 with 256 threads, 553 with 512).  Fewer: blocks
// of 512, and up to eight of them in a cluster share a row.
template <typename T>
static int launch_logp(const LogpParams& p, cudaStream_t s) {
  if (p.V <= 1024) return launch_logp_as<T, 32>(p, 1, s);
  if (p.M >= 8 * sm_count()) return launch_logp_as<T, 128>(p, 1, s);
  int ranks = 1;
  while (ranks < LP_MAX_RANKS && (long long)p.M * ranks * 2 <= 2ll * sm_count() && p.V / (ranks * 2) >= 2048) ranks *= 2;
  return launch_logp_as<T, 512>(p, ranks, s);
}

template <typename T>
static int launch_logp_bwd(const LogpBwdParams& p, cudaStream_t s) {
  // 16-byte accesses need every row of logits and gradient to start at the same offset from a 16-byte boundary
  const long long off = (long long)((uintptr_t)p.logits & 15) - (long long)((uintptr_t)p.dlogits & 15);
  const bool vec = off == 0 && ((p.ld - p.ld_d) * (long long)sizeof(T)) % 16 == 0;
  const int per = vec ? LB_THREADS * LB_VECS * Vec16<T>::N : LB_THREADS * 8;
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
  if (!sizes_ok(n, vocab) || d > PCM_MAX_VOCAB_CALL) return PCM_ERR_SHAPE;       // a thread's columns are counted in 32 bits
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
  if (n < 0 || vocab < 1 || d < 1 || d > PCM_MAX_EMBED_DIM || !sizes_ok(n, vocab)) return 0;
  EmbedPlan pl;
  return embed_plan(pl, n, vocab, d, nullptr) + 256;
}

extern "C" int grpo_embed_bwd(int32_t dtype, const void* dout, int64_t ld_dout, const int32_t* tok, int32_t n, int32_t vocab,
                              int32_t d, float scale, uint32_t flags, float* grad, uint32_t* device_status, void* workspace,
                              size_t workspace_bytes, pcm_stream stream) {
  if (!dtype_ok(dtype) || n < 0 || vocab < 1 || d < 1 || ld_dout < d || !std::isfinite(scale) || !grad) return PCM_ERR_ARG;
  if (((uintptr_t)grad & 3) || (flags & ~GRPO_ACCUMULATE)) return PCM_ERR_ARG;
  if (d > PCM_MAX_EMBED_DIM || !sizes_ok(n, vocab)) return PCM_ERR_SHAPE;
  cudaStream_t s = (cudaStream_t)stream;
  const bool accumulate = flags & GRPO_ACCUMULATE;
  if (n == 0) {
    if (!accumulate) PCM_CUDA_TRY(cudaMemsetAsync(grad, 0, (size_t)vocab * d * sizeof(float), s));
    return PCM_OK;
  }
  if (!dout || !tok || !elem_aligned(dout, dtype)) return PCM_ERR_ARG;
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < grpo_embed_workspace_bytes(n, vocab, d)) return PCM_ERR_WORKSPACE;
  prof_begin(PC_EMBED, s);
  const EmbedPlan pl = embed_sorted_plan(n, vocab, d, workspace);
  int rc = launch_embed_sort(pl, tok, device_status, s);
  if (rc == PCM_OK)
    rc = dtype == GRPO_BF16 ? launch_embed_sum(pl, (const __nv_bfloat16*)dout, ld_dout, nullptr, scale, accumulate, grad, s)
                            : launch_embed_sum(pl, (const float*)dout, ld_dout, nullptr, scale, accumulate, grad, s);
  prof_end(s, 2.0 * n * d, (double)n * d * (dtype == GRPO_BF16 ? 2.0 : 4.0) + 4.0 * vocab * d);
  return rc;
}

extern "C" int grpo_token_logp(int32_t dtype, const void* logits, int64_t ld, int32_t n_rows, int32_t vocab, const int32_t* tok,
                               float temperature, int32_t top, float* logp, float* entropy, float* lse, int32_t* top_id,
                               float* top_logp, uint32_t* device_status, pcm_stream stream) {
  if (!dtype_ok(dtype) || n_rows < 0 || vocab < 1 || ld < vocab || top < 0) return PCM_ERR_ARG;
  if (!vocab_temperature_ok(temperature)) return PCM_ERR_ARG;
  if (top > PCM_MAX_TOP || top > vocab || !sizes_ok(n_rows, vocab)) return PCM_ERR_SHAPE;
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
  if (!vocab_temperature_ok(temperature)) return PCM_ERR_ARG;
  if (!sizes_ok(n_rows, vocab)) return PCM_ERR_SHAPE;
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
