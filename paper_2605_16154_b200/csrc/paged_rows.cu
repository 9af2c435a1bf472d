// Attention of few new tokens over a paged cache in bf16: decoding steps, short chunks, and head dim 32.
//
// What bounds it is the reading of the cache, each key and value once for the 16 or 32 rows of a unit (new tokens times the
// query heads of a key-value head).  Four warps share a tile of 64 or 128 keys, and run through their unit without
// waiting for one another: each copies its own keys and values ahead into its own ring of shared memory (TMA, whose one
// instruction for 8 or 16 keys of a page leaves the warp's time to the products: with 16 bytes a lane a step of 256 sequences took
// 322 us), forms scores and weights in registers (mma.sync m16n8k16: a tile of so few rows would leave a tcgen05 tile of
// 128 rows nearly empty, and the products take a fraction of the time of the loads), and keeps its own running maximum, sum
// and values.  The warps' sums meet at the unit's end.  The weights enter the product with v
// as a pair of bf16 values, high and low part, so that they are not rounded: the second product hides behind the loads too.
// A step of 256 sequences of 500 to 8192 tokens, 16/4 heads of 128, takes 252 us (6.0 TB/s), of two of 131072, 32/8 heads, 158 us, of 256 of
// 300 tokens, 16 heads of 64, 90 us (3.5 TB/s: units of three tiles); one of 300 tokens
// 12 us, which are launches, dependent reads (lengths, table, keys) and the join.
#include <cuda.h>

#include "async_ptx.cuh"
#include "paged_attention.cuh"

namespace pcm {
namespace pga {

constexpr int RB_WARPS = 4, RB_THREADS = RB_WARPS * 32;
template <int DH> struct RbCfg {
  // keys of a warp's step: 8 KB of keys and values (4 at head dim 32), so that what a step costs beside them weighs alike
  static constexpr int KEYS = DH == 128 ? 16 : 32, TILE = RB_WARPS * KEYS;
  static constexpr int STAGES = DH == 32 ? 6 : 3;
  static constexpr int ROW = DH * 2, HALF = KEYS * ROW, STAGE = 2 * HALF;          // bytes: a key, a step's keys, keys and values
  static constexpr int RING = STAGES * STAGE;
  static constexpr int SLAB_COLS = DH < 64 ? DH : 64, SLABS = DH / SLAB_COLS;      // columns of a swizzled row
  static constexpr int SLAB_ROW = SLAB_COLS * 2, SLAB = KEYS * SLAB_ROW;
  static constexpr int BYTES = RB_WARPS * RING + 1024;             // tiles start on multiples of 1024 bytes
};

constexpr unsigned long long RB_WAIT_NS = 2000000000ull;
__device__ __forceinline__ void rb_load_4d(void* dst, const void* tmap, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
          smem_u32(dst)),
      "l"(tmap), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
__device__ __forceinline__ void rb_fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16-byte chunk c of row r within a step's rows of DH values, as TMA leaves them: eight rows of one chunk never share banks
template <int DH> __device__ __forceinline__ uint32_t rb_at(int r, int c) {
  using C = RbCfg<DH>;
  if (DH < 64) return (uint32_t)(r * C::SLAB_ROW + ((c ^ ((r >> 1) & 3)) << 4));
  return (uint32_t)((c >> 3) * C::SLAB + r * C::SLAB_ROW + (((c & 7) ^ (r & 7)) << 4));
}
// high and low bf16 parts of two weights
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  const __nv_bfloat162 l = __floats2bfloat162_rn(a - __low2float(h), b - __high2float(h));
  hi = *reinterpret_cast<const uint32_t*>(&h);
  lo = *reinterpret_cast<const uint32_t*>(&l);
}

template <int DH, int MT>
__global__ void __launch_bounds__(RB_THREADS, 2) attn_rows_bf16_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ AttnParams p,
                      const int box_rows) {
  using C = RbCfg<DH>;
  constexpr int UR = 16 * MT, KT = DH / 16, NT = DH / 8, LEAD = C::STAGES - 1;
  constexpr int KEYS = C::KEYS, NK = KEYS / 8, KB = KEYS / 16;     // keys of a step, in columns of 8 and blocks of 16
  extern __shared__ uint8_t rb_raw[];
  __shared__ Piece piece;
  __shared__ uint64_t full[RB_WARPS][C::STAGES];
  __shared__ float all_m[RB_WARPS][UR], all_l[RB_WARPS][UR], row_m[UR], row_l[UR];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  uint8_t* rb_smem = rb_raw + ((1024u - (smem_u32(rb_raw) & 1023u)) & 1023u);
  uint8_t* my_ring = rb_smem + warp * C::RING;
  const uint32_t ring = smem_u32(my_ring);
  if (lane == 0) {
    for (int i = 0; i < C::STAGES; ++i) mbar_init(&full[warp][i], 1);
    fence_mbar_init();
    prefetch_tmap(&tm_k);
    prefetch_tmap(&tm_v);
  }
  __syncwarp();
  unsigned asked = 0, taken = 0;               // steps copied into the ring and taken from it, over all units
  bool ok = true;

  wait_for_predecessor();
  block_piece(p, rb_smem, &piece);
  rb_fence_async();                            // what it needed of the ring goes to the copies
  __syncthreads();
  Cursor c = piece.c;
  long long left = piece.left, ahead = piece.ahead;
  const long long share = piece.share;
  int4 job = make_int4(0, 0, 0, -1);
  int redo = 0;

  while (left > 0) {
    const int t0 = c.at, t1 = (int)min((long long)c.u.tiles, t0 + left), steps = t1 - t0;
    const bool whole = t0 == 0 && t1 == c.u.tiles;
    auto first_key = [&](int i) {
      const int t = t0 + i;
      return (t < c.u.first_tiles ? t : t + c.u.skip) * C::TILE + warp * KEYS;
    };
    // Where the boxes of step i lie (lane: box): page and slot.  Boxes that no row of the unit sees lie behind the last page,
    // which reads as zeros.
    auto locate = [&](int i) {
      int2 at = make_int2(p.c.n_pages, 0);
      if (i < steps) {
        const int key = first_key(i) + lane * box_rows;
        if (lane * box_rows < KEYS && key < c.u.end && (key + box_rows > c.u.low || key < p.sinks)) {
          const int n = fast_div(key, p.c.div_page), page = p.c.table[c.s * p.c.ld_table + n];
          if (page >= 0 && page < p.c.n_pages) at = make_int2(page, key - n * p.c.page_size);
          else kv_report(p.c, STATUS_BAD_PAGE);
        }
      }
      return at;
    };
    auto copy = [&](int i, int2 at) {
      if (i >= steps || first_key(i) >= c.u.end || !ok) return;    // the same in all lanes
      const int st = asked % C::STAGES;
      uint64_t* bar = &full[warp][st];
      if (lane == 0) mbar_expect_tx(bar, C::STAGE);
      __syncwarp();
      if (lane * box_rows < KEYS) {
        uint8_t* dst = my_ring + st * C::STAGE + lane * box_rows * C::SLAB_ROW;
#pragma unroll
        for (int slab = 0; slab < C::SLABS; ++slab) {
          rb_load_4d(dst + slab * C::SLAB, &tm_k, slab * 64, c.head, at.y, at.x, bar);
          rb_load_4d(dst + C::HALF + slab * C::SLAB, &tm_v, slab * 64, c.head, at.y, at.x, bar);
        }
      }
      ++asked;
    };
#pragma unroll 1
    for (int i = 0; i < LEAD; ++i) copy(i, locate(i));
    int2 at_next = locate(LEAD);

    uint32_t qf[MT][KT][4];
    int pos[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const RowPlace x = row_place(p, c.sp, c.qt, c.head, mt * 16 + h * 8 + g);
        pos[mt][h] = x.pos;
        const __nv_bfloat16* q = (const __nv_bfloat16*)p.q + x.row * p.ld_q + x.head * p.ld_q_head + t4 * 2;
#pragma unroll
        for (int k = 0; k < KT; ++k) {
          qf[mt][k][h] = x.valid ? *reinterpret_cast<const uint32_t*>(q + k * 16) : 0u;
          qf[mt][k][2 + h] = x.valid ? *reinterpret_cast<const uint32_t*>(q + k * 16 + 8) : 0u;
        }
      }
    const int p_low = row_place(p, c.sp, c.qt, c.head, 0).pos, p_high = c.u.end - 1;

    float o[MT][NT][4], m[MT][2], l[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt][0] = m[mt][1] = -INFINITY;
      l[mt][0] = l[mt][1] = 0.f;
#pragma unroll
      for (int n = 0; n < NT; ++n) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.f;
    }
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
      copy(i + LEAD, at_next);
      at_next = locate(i + LEAD + 1);
      const int key0 = first_key(i);
      if (key0 < c.u.end && ok) {
        const int st = taken % C::STAGES;
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(&full[warp][st], (taken / C::STAGES) & 1u, RB_WAIT_NS));
        if (!ok) {                             // (the copies have not landed: the block's results are not meaningful)
          kv_report_expired(p.c);
          break;
        }
        ++taken;
        const uint32_t kb_at = ring + st * C::STAGE, vb = kb_at + C::HALF;
        if (key0 + KEYS > c.sp.len) {          // slots behind the end of a sequence may never have been written
          for (int r = max(0, c.sp.len - key0) * NT + lane; r < KEYS * NT; r += 32)
            *reinterpret_cast<uint4*>(my_ring + st * C::STAGE + C::HALF + rb_at<DH>(r / NT, r % NT)) = make_uint4(0, 0, 0, 0);
          rb_fence_async();
          __syncwarp();
        }
        float z[MT][NK][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int n = 0; n < NK; ++n) z[mt][n][0] = z[mt][n][1] = z[mt][n][2] = z[mt][n][3] = 0.f;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            uint32_t b[4];
            ldm4(b, kb_at + rb_at<DH>(kb * 16 + (lane & 7) + ((lane >> 4) << 3), k * 2 + ((lane >> 3) & 1)));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              mma16816(z[mt][2 * kb], qf[mt][k], b[0], b[1]);
              mma16816(z[mt][2 * kb + 1], qf[mt][k], b[2], b[3]);
            }
          }
        const bool all_seen = key0 + KEYS - 1 <= p_low &&
                              (p.window == 0 || key0 > p_high - p.window || key0 + KEYS - 1 < p.sinks);
        if (!all_seen)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (!row_sees(p, pos[mt][e >> 1], key0 + n * 8 + t4 * 2 + (e & 1))) z[mt][n][e] = -INFINITY;
        float top[MT][2];
        bool rise = false;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            top[mt][h] = fmaxf(z[mt][0][h * 2], z[mt][0][h * 2 + 1]);
#pragma unroll
            for (int n = 1; n < NK; ++n) top[mt][h] = fmaxf(top[mt][h], fmaxf(z[mt][n][h * 2], z[mt][n][h * 2 + 1]));
          }
#pragma unroll
        for (int d = 1; d <= 2; d <<= 1)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) top[mt][h] = fmaxf(top[mt][h], __shfl_xor_sync(0xffffffffu, top[mt][h], d));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) rise |= top[mt][0] > m[mt][0] || top[mt][1] > m[mt][1];
        if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float to = fmaxf(m[mt][h], top[mt][h]), f = to == -INFINITY ? 1.f : ex2((m[mt][h] - to) * p.scale_log2);
              m[mt][h] = to;
              l[mt][h] *= f;
#pragma unroll
              for (int n = 0; n < NT; ++n) { o[mt][n][h * 2] *= f; o[mt][n][h * 2 + 1] *= f; }
            }
        }
        uint32_t hi[MT][KB][4], lo[MT][KB][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float ref = m[mt][h] == -INFINITY ? 0.f : m[mt][h];
#pragma unroll
            for (int n = 0; n < NK; ++n) {
              const float a = ex2((z[mt][n][h * 2] - ref) * p.scale_log2), b = ex2((z[mt][n][h * 2 + 1] - ref) * p.scale_log2);
              l[mt][h] += a + b;
              split2(a, b, hi[mt][n >> 1][(n & 1) * 2 + h], lo[mt][n >> 1][(n & 1) * 2 + h]);
            }
          }
        // high parts of four columns of tiles, then their low parts: products into one accumulator wait for one another
#pragma unroll
        for (int n = 0; n < NT; n += 4)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            uint32_t b[2][4];
            ldm4t(b[0], vb + rb_at<DH>(kb * 16 + (lane & 7) + (((lane >> 3) & 1) << 3), n + (lane >> 4)));
            ldm4t(b[1], vb + rb_at<DH>(kb * 16 + (lane & 7) + (((lane >> 3) & 1) << 3), n + 2 + (lane >> 4)));
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  mma16816(o[mt][n + k], part ? lo[mt][kb] : hi[mt][kb], b[k >> 1][(k & 1) * 2], b[k >> 1][(k & 1) * 2 + 1]);
          }
      }
      __syncwarp();                            // the stage is copied over in the next step
    }
    // join the warps
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float s = l[mt][h];
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        if (t4 == 0) { all_m[warp][mt * 16 + h * 8 + g] = m[mt][h]; all_l[warp][mt * 16 + h * 8 + g] = s; }
      }
    __syncthreads();                           // every warp is through with its ring, which takes its sums now
    float* sums = reinterpret_cast<float*>(rb_smem);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<float2*>(sums + (warp * UR + mt * 16 + h * 8 + g) * DH + n * 8 + t4 * 2) = make_float2(o[mt][n][h * 2], o[mt][n][h * 2 + 1]);
    if (tid < UR) {
      float top = -INFINITY, sum = 0.f;
      for (int w = 0; w < RB_WARPS; ++w) top = fmaxf(top, all_m[w][tid]);
      const float ref = top == -INFINITY ? 0.f : top;
      for (int w = 0; w < RB_WARPS; ++w) {
        const float f = ex2((all_m[w][tid] - ref) * p.scale_log2);
        sum = fmaf(all_l[w][tid], f, sum);
        all_m[w][tid] = f;
      }
      row_m[tid] = top; row_l[tid] = sum;
    }
    __syncthreads();
    const int slot = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);
    float* part = p.part + (long long)slot * UR * DH;
    __nv_bfloat16* out = (__nv_bfloat16*)p.out;
    for (int i = tid * 2; i < UR * DH; i += RB_THREADS * 2) {
      const int r = i / DH, e = i - r * DH;
      const RowPlace x = row_place(p, c.sp, c.qt, c.head, r);
      if (!x.valid) continue;
      float a = 0.f, b = 0.f;
#pragma unroll
      for (int w = 0; w < RB_WARPS; ++w) {
        const float2 v = *reinterpret_cast<const float2*>(sums + w * UR * DH + i);
        a = fmaf(all_m[w][r], v.x, a);
        b = fmaf(all_m[w][r], v.y, b);
      }
      if (!whole) {
        *reinterpret_cast<float2*>(part + i) = make_float2(a, b);
      } else {
        const float inv = row_l[r] == 0.f ? 0.f : 1.f / row_l[r];
        *reinterpret_cast<__nv_bfloat162*>(out + x.row * p.ld_out + x.head * p.ld_out_head + e) = __floats2bfloat162_rn(a * inv, b * inv);
        redo |= !(isfinite(a) && isfinite(b)) && isfinite(row_l[r]);
      }
    }
    if (tid < UR) {
      const RowPlace x = row_place(p, c.sp, c.qt, c.head, tid);
      if (!whole) p.part_ml[(long long)slot * UR + tid] = make_float2(row_m[tid], row_l[tid]);
      else if (x.valid && p.lse)
        p.lse[x.row * p.n_heads + x.head] = row_l[tid] == 0.f ? -INFINITY : fmaf(row_m[tid], p.scale_log2, log2f(row_l[tid])) * LN2;
    }
    rb_fence_async();                          // the ring goes back from sums to copies
    __syncthreads();
    if (!whole && t0 == 0) job = make_int4(c.s, c.qt, c.head, last_worker(p, blockIdx.x, share, ahead, c.u.tiles));
    left -= steps;
    ahead += steps;
    if (left > 0) c.next_unit(p);
  }
  if (!ok)                                     // nothing may land after the block is gone
    for (; taken < asked; ++taken) mbar_wait_bounded(&full[warp][taken % C::STAGES], (taken / C::STAGES) & 1u, RB_WAIT_NS / 8);
  redo = __syncthreads_or(redo);
  if (tid == 0) { p.jobs[blockIdx.x] = job; p.redo[blockIdx.x] = redo; p.pieces[blockIdx.x] = piece; }
  let_successor_start();
}

template <int DH, int MT>
static int launch_rows(const AttnParams& p, cudaStream_t s) {
  static std::atomic<unsigned long long> seen{0};
  if (const int rc = allow_smem(attn_rows_bf16_kernel<DH, MT>, RbCfg<DH>::BYTES, &seen)) return rc;
  int box = RbCfg<DH>::KEYS;
  while (p.c.page_size % box) box /= 2;        // (pages are of a multiple of 8)
  CUtensorMap tm_k, tm_v;
  if (!page_map(&tm_k, p.c.k, p.c, DH, RbCfg<DH>::SLAB_COLS, box) || !page_map(&tm_v, p.c.v, p.c, DH, RbCfg<DH>::SLAB_COLS, box)) return PCM_ERR_CUDA;
  return launch_after_smem(attn_rows_bf16_kernel<DH, MT>, dim3(p.workers), dim3(RB_THREADS), RbCfg<DH>::BYTES, s, tm_k, tm_v, p, box);
}
int attn_rows_tile(int dh) { return dh == 128 ? RbCfg<128>::TILE : dh == 64 ? RbCfg<64>::TILE : RbCfg<32>::TILE; }
int launch_rows_bf16(const AttnParams& p, int dh, cudaStream_t s) {
  if (p.unit_rows == 16) return dh == 128 ? launch_rows<128, 1>(p, s) : dh == 64 ? launch_rows<64, 1>(p, s) : launch_rows<32, 1>(p, s);
  if (dh == 128) return PCM_ERR_SHAPE;          // (16 rows are all that its registers hold)
  return dh == 64 ? launch_rows<64, 2>(p, s) : launch_rows<32, 2>(p, s);
}

}  // namespace pga
}  // namespace pcm
