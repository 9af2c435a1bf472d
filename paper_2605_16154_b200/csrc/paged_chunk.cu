// Attention of chunks of new tokens over a paged cache in bf16, head dims 64 and 128, on the fifth-generation tensor cores.
//
// A unit is 256 rows in two streams of 128; the keys come in tiles of 128.  Per stream and tile:
//   S = Q K^T            tcgen05.mma, 128 x 128 fp32 in tensor memory
//   P = 2^(c S - c m)    four softmax warps, a thread per row: the weights are packed to bf16 over the scores they came from
//   O += P V             tcgen05.mma with P from tensor memory, accumulated there
// While one stream's warps form weights the tensor core works for the other.  The streams have an issuing warp each and run
// at their own pace, a ring of tiles apart at most; from unit to unit they change halves, since the later half sees more.  The
// reference m of a row is the first score that it sees, and it moves only when a tile's maximum has risen by more than 32 powers
// of two above it, to that maximum from the next tile on: weights far above 1 are as exact in bf16 and fp32 as weights up to 1,
// the accumulator is hardly ever fetched, scaled and put back, and no weight waits for the maximum of its tile.  A tile that rises by more than 100
// powers of two at once (70 nats) has its rows formed once more where pieces are joined: right, but by single warps, key by key (every
// row of 1024 behind 4096, 16/4 heads of 128: 26 ms instead of 0.08).  Rounding the weights to bf16 is what lets them be an operand of the
// tensor core; their sum is taken from the unrounded ones (error of the output 2.3e-3 of its norm, 1.7e-3 of it the output's own rounding).
// Keys and values come by TMA through a ring of tiles, box by box of a page (greatest common divisor of page and tile):
// lanes of the loading warp look their boxes' pages up side by side.  Boxes that no row of the unit sees are read from
// behind the last page, which yields zeros: what the table says there does not matter.  Value rows behind the end of a sequence
// are cleared in shared memory, since a page may never have been written there.
//
// Warps 0-3 and 4-7: softmax and output of streams 0 and 1.  Warps 8 and 10: products of streams 0 and 1.  Warps 9 and 11: loads of
// keys and values.
//
// What bounds it is the latency from one product to the next: a tile of 256 rows takes about 4300 cycles where the tensor pipe and
// the exponential unit need 2048 each (44 to 47 % busy).  8 x 1024 tokens behind 4096 to 8192, 16/4 heads of 128: 385 us, 868 TFLOP/s,
// and 410 to 425 once the clock falls under a row of such calls; 384 prefixes of 256, 16 heads of 64: 248 us, 0.81 GB at 3.3 TB/s, where
// the change of units costs as much as its tiles.
// Every wait is bounded; one that expires is reported in the call's status word, or the device's, and ends the block.
#include <cuda.h>

#include "async_ptx.cuh"
#include "paged_attention.cuh"
#include "tensor_map.h"

namespace pcm {
namespace pga {

constexpr int CH_ROWS = 128, CH_TILE = 128, CH_THREADS = 384;
constexpr unsigned long long CH_WAIT_NS = 2000000000ull;
constexpr int CH_TMEM = 512;
// Tiles of a piece from which on its streams take turns at head dim 128, whose products keep the tensor core as busy as the exponential
// unit (8 x 1024 tokens, 16/4 heads, the last of 128 x 16 keys: 158 us, 166 without; x 32: 302, 319; x 96: 962, 1014; 37 x 16 heads of 256
// tokens, x 24: 319, 322; below 12 tiles the same; two tiles: 4 % more).  At head dim 64 the exponential unit sets the pace and turns cost 6 to 15 % (x 16: 139 us, 122
// without; x 32: 259, 225; x 96: 756, 641).
constexpr int CH_TURNS = 8;
constexpr int CH_TURN_TRIES = 1 << 12;
constexpr float CH_RISE = 32.f;                // powers of two by which a maximum may outgrow its reference
constexpr float CH_WILD = 100.f;               // .. within one tile: 128 weights of 2^100 still have a sum
template <int DH> struct ChCfg {
  static constexpr int SLABS = DH / 64;        // 64 columns of 128 rows, 128-byte swizzle
  static constexpr int SLAB = 128 * 128, TILE_BYTES = SLABS * SLAB;
  static constexpr int STAGES = DH == 128 ? 5 : 8;
  static constexpr int QBUFS = DH == 128 ? 1 : 2;                  // a stream's queries: the next unit's beside this one's where they fit
  static constexpr int RING_AT = 2 * QBUFS * TILE_BYTES, BAR_AT = RING_AT + STAGES * TILE_BYTES;
  static constexpr int SMALL_AT = BAR_AT + 512, BYTES = SMALL_AT + 1024;
  static_assert(BYTES <= 227 * 1024, "shared memory");
  static constexpr int O_COL = 256;            // scores of the streams: columns 0 and 128; values: from 256 on
};

// Issued by one lane of a converged warp (`me`): operands that the whole warp agrees on stay in uniform registers, which these
// instructions read; in code of a single lane each operand is moved there one by one (about 100 cycles a product).
__device__ __forceinline__ int ch_elect() {
  int e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e;
}
__device__ __forceinline__ void ch_load_4d(int me, void* dst, const void* tmap, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %7, 0;\n\t"
      "@e cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];\n\t}" ::"r"(
          smem_u32(dst)),
      "l"(tmap), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(me)
      : "memory");
}
__device__ __forceinline__ void ch_mma_ss(int me, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(me)
      : "memory");
}
__device__ __forceinline__ void ch_mma_ts(int me, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(me)
      : "memory");
}
__device__ __forceinline__ void ch_commit(int me, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %1, 0;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"(me)
      : "memory");
}
__device__ __forceinline__ void ch_tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ float ch_tmem_ld1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(r) : "r"(taddr) : "memory");
  return __uint_as_float(r);
}
__device__ __forceinline__ void ch_tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// Loads are over, and what they bring is not read before.
__device__ __forceinline__ void ch_ld_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                 "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                 "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
__device__ __forceinline__ void ch_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void ch_fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ uint64_t ch_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  return (uint64_t)((saddr >> 4) & 0x3FFF) | (uint64_t)((lbo >> 4) & 0x3FFF) << 16 | (uint64_t)((sbo >> 4) & 0x3FFF) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// fp32 accumulator, bf16 operands, M = 128
__device__ __forceinline__ uint32_t ch_idesc(int n, int b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(d))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
        "l"(reinterpret_cast<unsigned long long&>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(d))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ void ch_copy16(void* dst, const void* src, bool take) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ch_copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ uint32_t ch_pack(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Waits for a phase until it completes, the block gives up, or two seconds have passed (then it gives up for the block).
__device__ __forceinline__ bool ch_wait(uint64_t* bar, unsigned parity, volatile unsigned* gave_up, const KvView& c) {
  if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long from = global_timer_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*gave_up) return false;
    if (global_timer_ns() - from > CH_WAIT_NS) {
      *gave_up = 1;
      kv_report_expired(c);
      return false;
    }
  }
}

// The positions of the rows of half h of a unit.
struct ChStream { int lo, hi; bool rows; };
__device__ __forceinline__ ChStream ch_stream(const AttnParams& p, const SeqSpan& sp, int qt, int h) {
  ChStream x;
  const int total = sp.fresh * p.group, r0 = qt * 2 * CH_ROWS + h * CH_ROWS;
  x.rows = r0 < total;
  const int r1 = min(total, r0 + CH_ROWS) - 1, first = sp.len - sp.fresh;
  x.lo = x.rows ? first + fast_div(r0, p.div_group) : -1;
  x.hi = x.rows ? first + fast_div(r1, p.div_group) : -1;
  return x;
}
__device__ __forceinline__ int ch_key(const UnitSpan& u, int i) { return (i < u.first_tiles ? i : i + u.skip) * CH_TILE; }
// Which of tiles [t0, t1) of the unit the rows see: [t0, a) for the first tokens, [b, e) for those before a row.
struct ChRange { int t0, a, b, e; };
__device__ __forceinline__ ChRange ch_range(const AttnParams& p, const ChStream& x, const UnitSpan& u, int t0, int t1) {
  auto index = [&](int tile) { return tile <= u.first_tiles ? tile : max(u.first_tiles, tile - u.skip); };     // first index from this tile on
  ChRange r;
  r.t0 = t0;
  r.e = x.rows && x.hi >= 0 ? max(t0, min(t1, index(x.hi / CH_TILE + 1))) : t0;
  r.a = t0;
  r.b = t0;
  if (p.window > 0) {
    r.a = max(t0, min(r.e, index((p.sinks + CH_TILE - 1) / CH_TILE)));
    r.b = max(r.a, min(r.e, index(x.lo >= p.window ? (x.lo - p.window + 1) / CH_TILE : 0)));
  }
  return r;
}
// The same within tiles [t0, t1) only.
__device__ __forceinline__ ChRange ch_clip(const ChRange& r, int t0, int t1) {
  ChRange x;
  x.t0 = t0;
  x.a = max(t0, min(r.a, t1));
  x.b = max(x.a, min(r.b, t1));
  x.e = max(x.b, min(r.e, t1));
  return x;
}
// What the two halves of a unit see; the heads of a row tile have it in common.
struct ChSight {
  int s, qt;
  ChRange r[2];
  __device__ void learn(const AttnParams& p, const Cursor& c) {
    if (c.s == s && c.qt == qt) return;
    s = c.s; qt = c.qt;
    r[0] = ch_range(p, ch_stream(p, c.sp, c.qt, 0), c.u, 0, c.u.tiles);
    r[1] = ch_range(p, ch_stream(p, c.sp, c.qt, 1), c.u, 0, c.u.tiles);
  }
  __device__ ChRange of(int half, int t0, int t1) const {
    ChRange x = r[0];
    if (half) x = r[1];
    return ch_clip(x, t0, t1);
  }
};
__device__ __forceinline__ bool ch_in(const ChRange& r, int i) { return i < r.a || (i >= r.b && i < r.e); }
__device__ __forceinline__ bool ch_any(const ChRange& r) { return r.a > r.t0 || r.b < r.e; }

struct ChBars {
  uint64_t full[10], empty[10];                // tiles of the ring
  uint64_t landed;                             // a tile that is cleaned before it is handed on
  int filled[10];                              // what the tiles wait for should the block give up: 1 + the last ring position ..
  int cleaning;                                // .. and 1 + the phase of `landed`, 0: nothing
  uint64_t q_full[2], s_full[2], p_half[2], p_full[2], o_full[2], done[2];
  uint32_t tmem;
  unsigned gave_up;
  unsigned turn[4];                            // 1: a warp of this quarter of the SM forms weights
  int redo;
};

template <int DH>
__global__ void __launch_bounds__(CH_THREADS, 1)
attn_chunk_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ AttnParams p,
                  const int box_rows) {
  using C = ChCfg<DH>;
  extern __shared__ __align__(1024) uint8_t ch_smem[];             // a swizzled tile starts on a multiple of 1024 bytes
  struct Small {
    Piece piece;
    Cursor coming[8];        // each softmax warp's next unit, where its queries are asked for ahead of time
  };
  uint8_t* base = ch_smem;
  Small& sh = *reinterpret_cast<Small*>(base + C::SMALL_AT);
  static_assert(sizeof(Small) <= C::BYTES - C::SMALL_AT, "shared memory");
  ChBars& b = *reinterpret_cast<ChBars*>(base + C::BAR_AT);
  static_assert(sizeof(ChBars) <= 512, "barriers");
  volatile unsigned* gave_up = &b.gave_up;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < C::STAGES; ++i) { mbar_init(&b.full[i], 1); mbar_init(&b.empty[i], 2); }
    mbar_init(&b.landed, 1);
    for (int s = 0; s < 2; ++s) { mbar_init(&b.q_full[s], 4); mbar_init(&b.s_full[s], 1); mbar_init(&b.p_half[s], 4); mbar_init(&b.p_full[s], 4); mbar_init(&b.o_full[s], 1); mbar_init(&b.done[s], 1); }
    b.gave_up = 0;
    b.cleaning = 0;
    for (int i = 0; i < C::STAGES; ++i) b.filled[i] = 0;
    for (int i = 0; i < 4; ++i) b.turn[i] = 0;
    b.redo = 0;
    fence_mbar_init();
    prefetch_tmap(&tm_k);
    prefetch_tmap(&tm_v);
  }
  if (warp == 8) {
    tmem_alloc(&b.tmem, CH_TMEM);
    tmem_relinquish();
  }
  wait_for_predecessor();
  block_piece(p, base + C::RING_AT, &sh.piece);
  ch_fence_async();                            // what it needed of the ring goes to the copies
  if (tid == 0) p.pieces[blockIdx.x] = sh.piece;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = b.tmem;
  Cursor c = sh.piece.c;
  long long left = sh.piece.left;

  if (warp >= 8) {
    if (warp == 9 || warp == 11) {
      // ---------------------------- loads: keys and values, a warp each ----------------------------
      // The ring takes K0 K1 V0 K2 V1 .., as the products want them.
      const bool values = warp == 11;
      const int me = ch_elect(), boxes = CH_TILE / box_rows;
      const void* tm = values ? &tm_v : &tm_k;
      unsigned landed_phase = 0;
      bool ok = true;
      int base_at = 0;                         // ring position of a piece's first keys
      // The page and slot of box `lane` of tile i.  Boxes that the unit does not see lie behind the last page.
      auto look_up = [&](int i, int& page, int& slot) {
        const int key = ch_key(c.u, i) + lane * box_rows;
        page = p.c.n_pages;
        slot = 0;
        if (lane < boxes && key < c.u.end && (key + box_rows > c.u.low || key < p.sinks)) {
          const int at = fast_div(key, p.c.div_page);
          page = p.c.table[c.s * p.c.ld_table + at];
          slot = key - at * p.c.page_size;
          if (page < 0 || page >= p.c.n_pages) { page = p.c.n_pages; kv_report(p.c, STATUS_BAD_PAGE); }
        }
      };
      while (left > 0 && ok) {
        const int t0 = c.at, t1 = (int)min((long long)c.u.tiles, t0 + left), n = t1 - t0;
        int page, slot;
        look_up(t0, page, slot);
        for (int i = 0; i < n; ++i) {
          const int at = base_at + (values ? (i + 1 < n ? 2 * i + 2 : 2 * i + 1) : i == 0 ? 0 : 2 * i - 1), st = at % C::STAGES;
          if (!__all_sync(0xffffffffu, ch_wait(&b.empty[st], ((unsigned)(at / C::STAGES) & 1u) ^ 1u, gave_up, p.c))) { ok = false; break; }
          uint8_t* dst = base + C::RING_AT + st * C::TILE_BYTES;
          const int key0 = ch_key(c.u, t0 + i);
          const bool clean = values && key0 + CH_TILE > c.sp.len;
          uint64_t* bar = clean ? &b.landed : &b.full[st];
          if (me) {
            if (clean) b.cleaning = 1 + (int)landed_phase;
            else b.filled[st] = at + 1;
            mbar_expect_tx(bar, C::TILE_BYTES);
          }
          __syncwarp();
          for (int k = 0; k < boxes; ++k) {
            const int page_k = __shfl_sync(0xffffffffu, page, k), slot_k = __shfl_sync(0xffffffffu, slot, k);
#pragma unroll
            for (int slab = 0; slab < C::SLABS; ++slab)
              ch_load_4d(me, dst + slab * C::SLAB + k * box_rows * 128, tm, slab * 64, c.head, slot_k, page_k, bar);
          }
          if (i + 1 < n) look_up(t0 + i + 1, page, slot);
          if (clean) {
            if (!__all_sync(0xffffffffu, ch_wait(&b.landed, landed_phase, gave_up, p.c))) { ok = false; break; }
            landed_phase ^= 1u;
            const int from = max(0, c.sp.len - key0);
            for (int r = from * C::SLABS * 8 + lane; r < CH_TILE * C::SLABS * 8; r += 32) {
              const int row = r / (C::SLABS * 8), part = r % (C::SLABS * 8);
              *reinterpret_cast<uint4*>(dst + (part >> 3) * C::SLAB + row * 128 + (part & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            ch_fence_async();
            __syncwarp();
            if (me) {
              b.cleaning = 0;
              b.filled[st] = at + 1;
              mbar_arrive(&b.full[st]);
            }
          }
        }
        base_at += 2 * n;
        left -= n;
        if (left > 0) c.next_unit(p);
      }
    } else {
      // ---------------------------- products of one stream ----------------------------
      const int s = warp == 8 ? 0 : 1, me = ch_elect();
      const uint64_t k0 = ch_desc(smem_u32(base + C::RING_AT), 16u, 1024u), v0 = ch_desc(smem_u32(base + C::RING_AT), C::SLAB, 1024u);
      const uint32_t q_lo = (uint32_t)ch_desc(smem_u32(base), 16u, 1024u), k_hi = (uint32_t)(k0 >> 32), v_hi = (uint32_t)(v0 >> 32);
      const uint32_t idesc_s = ch_idesc(CH_TILE, 0), idesc_o = ch_idesc(DH, 1);
      const uint32_t s_col = tmem + s * CH_TILE, o_col = tmem + C::O_COL + s * DH;
      auto desc = [](uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; };
      int k_at = 0, uses = 0, half = s;        // ring position of a piece's first keys; units with tiles so far
      unsigned p_phase = 0;
      bool ok = true;
      auto wait = [&](uint64_t* bar, unsigned parity) {
        if (ok && !__all_sync(0xffffffffu, ch_wait(bar, parity, gave_up, p.c))) ok = false;
        return ok;
      };
      auto ring_wait = [&](int n) { return wait(&b.full[n % C::STAGES], (unsigned)(n / C::STAGES) & 1u); };
      auto release = [&](int n, bool used) {
        if (used) ch_commit(me, &b.empty[n % C::STAGES]);
        else if (me) mbar_arrive(&b.empty[n % C::STAGES]);
      };
      auto scores = [&](int n, int q_buf) {
        const uint32_t qa = q_lo + (uint32_t)((s * C::QBUFS + q_buf) * (C::TILE_BYTES >> 4));
        const uint32_t ka = (uint32_t)k0 + (uint32_t)((n % C::STAGES) * (C::TILE_BYTES >> 4));
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < DH / 16; ++k) {
          const uint32_t o = (uint32_t)((k >> 2) * (C::SLAB >> 4) + (k & 3) * 2);
          ch_mma_ss(me, s_col, desc(qa + o, k_hi), desc(ka + o, k_hi), idesc_s, k > 0);
        }
        ch_commit(me, &b.s_full[s]);
      };
      ChSight sight;
      sight.s = -1;
      while (left > 0 && ok) {
        const int t0 = c.at, t1 = (int)min((long long)c.u.tiles, t0 + left);
        sight.learn(p, c);
        const ChRange r = sight.of(half, t0, t1);
        const bool any = __any_sync(0xffffffffu, ch_any(r));       // a half without tiles here brings no queries
        const int q_buf = uses % C::QBUFS;
        uint32_t begun = 0;
        if (!ring_wait(k_at)) break;
        if (any) {
          if (!wait(&b.q_full[s], (unsigned)uses & 1u)) break;
          ++uses;
        }
        bool now = __any_sync(0xffffffffu, ch_in(r, t0));
        if (now) scores(k_at, q_buf);
        release(k_at, now);
        for (int i = t0; i < t1; ++i) {
          // the ring holds K0 K1 V0 K2 V1 ..: the next tile's keys, then this one's values
          const bool more = i + 1 < t1, then = __any_sync(0xffffffffu, more && ch_in(r, i + 1));
          const int vn = k_at + (more ? 2 : 1);
          if (!ring_wait(vn)) break;
          if (now) {
            const uint32_t va = (uint32_t)v0 + (uint32_t)((vn % C::STAGES) * (C::TILE_BYTES >> 4));
            if (!wait(&b.p_half[s], p_phase)) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < CH_TILE / 32; ++k)
              ch_mma_ts(me, o_col, s_col + k * 8, desc(va + (uint32_t)(k * 128), v_hi), idesc_o, k > 0 ? 1u : begun);
            if (!wait(&b.p_full[s], p_phase)) break;
            p_phase ^= 1u;
            tc_fence_after();
#pragma unroll
            for (int k = CH_TILE / 32; k < CH_TILE / 16; ++k)
              ch_mma_ts(me, o_col, s_col + k * 8, desc(va + (uint32_t)(k * 128), v_hi), idesc_o, 1u);
            ch_commit(me, &b.o_full[s]);
            begun = 1;
          }
          if (more) {
            if (!ring_wait(k_at + 1)) break;
            if (then) scores(k_at + 1, q_buf);
            release(k_at + 1, then);
          }
          release(vn, now);
          k_at = more ? k_at + 2 : vn + 1;
          now = then;
        }
        left -= t1 - t0;
        half ^= 1;
        if (left > 0) c.next_unit(p);
      }
      ch_commit(me, &b.done[s]);               // every product is over before the block frees what they use
      mbar_wait_bounded(&b.done[s], 0, CH_WAIT_NS);
    }
  } else {
    // ---------------------------- weights and output: 128 threads a stream, a row each ----------------------------
    const int s = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t s_col = lanes + s * CH_TILE, o_col = lanes + C::O_COL + s * DH;
    unsigned s_phase = 0, o_count = 0;         // o_count: tiles whose weights have been handed over
    int uses = 0, half = s;                    // units whose queries have been asked for; the half of the unit at hand
    bool ok = true;
    if (tid == 0) p.jobs[blockIdx.x] = make_int4(0, 0, 0, -1);
    auto tiles_end = [](const Cursor& c, long long left) { return (int)min((long long)c.u.tiles, c.at + left); };
    ChSight sight;
    sight.s = -1;
    int q_buf = 0;                             // buffer of the queries at hand
    // A half's queries go to shared memory, 16 bytes a lane, as the products read them (128-byte swizzle); so do its values on
    // their way out.
    constexpr int PER = DH / 8;                // lanes a row
    auto tile_at = [&](int buf, int r, int ch) { return base + (s * C::QBUFS + buf) * C::TILE_BYTES + (ch >> 3) * C::SLAB + r * 128 + (((ch & 7) ^ (r & 7)) << 4); };
    auto ask_queries = [&](const Cursor& c, int h) {
      const RowPlace x = row_place(p, c.sp, c.qt, c.head, h * CH_ROWS + row);
      const long long mine = x.valid ? x.row * p.ld_q + x.head * p.ld_q_head : -1;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int r = i * (32 / PER) + lane / PER, ch = lane % PER;
        const long long from = __shfl_sync(0xffffffffu, mine, r);
        ch_copy16(tile_at(uses % C::QBUFS, quad * 32 + r, ch), (const __nv_bfloat16*)p.q + (from < 0 ? 0 : from + ch * 8), from >= 0);
      }
      ++uses;
    };
    auto hand_queries = [&]() {
      ch_copies_done();
      ch_fence_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.q_full[s]);
    };
    if (left > 0) {
      sight.learn(p, c);
      if (ch_any(sight.of(half, c.at, tiles_end(c, left)))) {
        ask_queries(c, half);
        hand_queries();
      }
    }
    while (left > 0 && ok) {
      const int t0 = c.at, t1 = tiles_end(c, left);
      const bool whole = t0 == 0 && t1 == c.u.tiles;
      const ChRange range = sight.of(half, t0, t1);
      const int pos = row_place(p, c.sp, c.qt, c.head, half * CH_ROWS + row).pos;
      const int w_lo = __shfl_sync(0xffffffffu, pos, 0), w_hi = __reduce_max_sync(0xffffffffu, pos);
      const bool turns = DH == 128 && range.e - range.b >= CH_TURNS;
      const long long rest = left - (t1 - t0);
      bool asked = false;
      if constexpr (C::QBUFS == 2) {           // the next unit's queries come in while this one's scores are formed
        Cursor next = c;
        if (rest > 0) {
          next.next_unit(p);
          sight.learn(p, next);
          asked = ch_any(sight.of(half ^ 1, next.at, tiles_end(next, rest)));
          if (asked) ask_queries(next, half ^ 1);
        }
        if (lane == 0) sh.coming[warp] = next;
        __syncwarp();
      }
      // the row's reference, what it is to be, the sum of its weights (a row ahead of every token waits for no reference)
      float m = pos < 0 ? 0.f : -INFINITY, m_next = m, l = 0.f;
      bool wild = false;                       // a tile rose so far above the reference that its weights may not fit
      bool begun = false;
      for (int i = t0;; ++i) {
        if (i == range.a) i = range.b;
        if (i >= range.e) break;
        const int key0 = ch_key(c.u, i);
        const bool all_seen = key0 + CH_TILE - 1 <= w_lo && (p.window == 0 || key0 > w_hi - p.window || key0 + CH_TILE - 1 < p.sinks);
        const bool none_yet = __any_sync(0xffffffffu, m == -INFINITY), rises = __any_sync(0xffffffffu, m_next != m);
        ok = __all_sync(0xffffffffu, ch_wait(&b.s_full[s], s_phase, gave_up, p.c));
        if (!ok) break;
        s_phase ^= 1u;
        tc_fence_after();
        // The warps run through more instructions a tile than are held close by, so loops stay loops: 64 scores a time (16 took 444 us
        // of far chunks, 32 423, 64 393).  Masks
        // are selects: a branch per score would cost ten times as much.
        const int last = pos - key0, from = pos - p.window + 1 - key0, sunk = p.sinks - key0;
        const bool behind = p.window > 0 && __any_sync(0xffffffffu, from > 0);
        auto mask = [&](uint32_t (&z)[32], int k0) {
#pragma unroll
          for (int e = 0; e < 32; ++e) z[e] = e > last - k0 ? 0xFF800000u : z[e];
          if (behind)
#pragma unroll
            for (int e = 0; e < 32; ++e) z[e] = (e < from - k0) & (e >= sunk - k0) ? 0xFF800000u : z[e];
        };
        // The reference of a tile's weights comes from the tiles before it, so that they need not wait for this one's maximum.
        if (none_yet) {
          // any score that the row sees will do: weights stay exact far above 1
          const float first = ch_tmem_ld1(s_col);
          if (m == -INFINITY && last >= 0 && !(p.window > 0 && from > 0 && sunk <= 0)) m = first;
          m_next = fmaxf(m_next, m);           // (other rows of the warp may be about to move theirs)
        }
        if (none_yet && __any_sync(0xffffffffu, m == -INFINITY && last >= 0)) {
          float tops[2] = {m, m};
#pragma unroll 1
          for (int k = 0; k < CH_TILE; k += 32) {
            uint32_t z[32];
            tmem_ld_32x32(s_col + k, z);
            tmem_ld_wait();
            if (!all_seen) mask(z, k);
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              tops[0] = max3(tops[0], __uint_as_float(z[e]), __uint_as_float(z[e + 1]));
              tops[1] = max3(tops[1], __uint_as_float(z[e + 2]), __uint_as_float(z[e + 3]));
            }
          }
          if (m == -INFINITY) m_next = m = fmaxf(tops[0], tops[1]);
        }
        if ((none_yet || rises) && begun && __any_sync(0xffffffffu, m_next != m)) {       // (the last tile's values are summed: these scores came after them)
          const float f = m_next > m ? ex2((m - m_next) * p.scale_log2) : 1.f;
#pragma unroll 1
          for (int k = 0; k < DH; k += 16) {
            uint32_t o[16];
            ch_tmem_ld16(o_col + k, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            ch_tmem_st16(o_col + k, o);
          }
          ch_tmem_st_wait();
          l *= f;
          if (m_next > m) m = m_next;
        }
        const float mc = m == -INFINITY ? 0.f : -m * p.scale_log2;
        const float2 c2 = make_float2(p.scale_log2, p.scale_log2), mc2 = make_float2(mc, mc);
        float2 sums[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        float tops[2] = {m, m};                // (a NaN shows in the sum of weights)
        // The two warps of a quarter of the SM, one of each stream, take turns: side by side both would end late, and the tensor
        // core would wait for both at once.
        if (turns) {
          if (lane == 0)                       // (a turn saves time and guards nothing: the wait for it may end)
            for (int n = 0; n < CH_TURN_TRIES && atomicCAS_block(&b.turn[quad], 0u, 1u) != 0u; ++n) {}
          __syncwarp();
        }
        auto hand_over = [&](int h) {
          ch_tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(h == 0 ? &b.p_half[s] : &b.p_full[s]);
        };
        auto form = [&](const uint32_t (&z)[32], int k) {          // weights of 32 keys, over scores that have been read
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float2 x0 = make_float2(__uint_as_float(z[e]), __uint_as_float(z[e + 1]));
            const float2 x1 = make_float2(__uint_as_float(z[e + 2]), __uint_as_float(z[e + 3]));
            float2 a = fma2(x0, c2, mc2), d = fma2(x1, c2, mc2);
            a.x = ex2(a.x);
            a.y = ex2(a.y);
            d.x = ex2(d.x);
            d.y = ex2(d.y);
            tops[0] = max3(tops[0], x0.x, x0.y);
            tops[1] = max3(tops[1], x1.x, x1.y);
            sums[0] = add2(sums[0], a);
            sums[1] = add2(sums[1], d);
            w[e >> 1] = ch_pack(a.x, a.y);
            w[(e >> 1) + 1] = ch_pack(d.x, d.y);
          }
          ch_tmem_st16(s_col + k * 16, w);
        };
        if (all_seen) {                        // 32 scores come in while 32 weights are formed
          uint32_t z[2][32];
          tmem_ld_32x32(s_col, z[0]);
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            ch_ld_wait(z[0]);
            tmem_ld_32x32(s_col + h * 64 + 32, z[1]);
            form(z[0], 2 * h);
            ch_ld_wait(z[1]);
            if (h == 0) tmem_ld_32x32(s_col + 64, z[0]);
            form(z[1], 2 * h + 1);
            hand_over(h);
          }
        } else {
#pragma unroll 1
          for (int k = 0; k < 4; ++k) {
            if (key0 + k * 32 > w_hi) {        // behind every row of the warp
              uint32_t none[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) none[e] = 0u;
              ch_tmem_st16(s_col + k * 16, none);
            } else {
              uint32_t z[32];
              tmem_ld_32x32(s_col + k * 32, z);
              tmem_ld_wait();
              if (key0 + k * 32 + 31 > w_lo || behind) mask(z, k * 32);
              form(z, k);
            }
            if (k & 1) hand_over(k >> 1);
          }
        }
        if (turns && lane == 0) atomicExch_block(&b.turn[quad], 0u);
        l += (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y);
        const float top = fmaxf(tops[0], tops[1]), over = (top - m) * p.scale_log2;
        m_next = over > CH_RISE ? top : m;
        if (over > CH_WILD || fabsf(mc) == INFINITY) wild = true;      // (a scaled reference beyond fp32 hides every difference from it)
        if (top == INFINITY) l = NAN;          // an infinite score makes its row NaN, like a NaN
        ++o_count;
        begun = true;
      }
      if (!ok) break;
      // every score of this piece is formed: its queries' place is free
      const RowPlace place = row_place(p, c.sp, c.qt, c.head, half * CH_ROWS + row);
      Cursor next = c;
      if constexpr (C::QBUFS == 2) {
        next = sh.coming[warp];
        __syncwarp();
        if (asked) hand_queries();
      }
      if (__any_sync(0xffffffffu, place.valid)) {
        if (begun) {
          ok = __all_sync(0xffffffffu, ch_wait(&b.o_full[s], (o_count - 1) & 1u, gave_up, p.c));
          if (!ok) break;
          tc_fence_after();
        }
        const int slot = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);
        const long long at = (long long)slot * p.unit_rows + half * CH_ROWS + row;
        const long long out_at = place.row * p.ld_out + place.head * p.ld_out_head;
        const float inv = wild ? NAN : l == 0.f ? 0.f : 1.f / l;
        float2 bad = make_float2(0.f, 0.f);    // NaN once a value is not finite
#pragma unroll 1
        for (int k = 0; k < DH; k += 32) {
          uint32_t o[32];
          if (begun) {
            tmem_ld_32x32(o_col + k, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0u;
          }
#pragma unroll
          for (int e = 0; e < 32; e += 2) bad = fma2(make_float2(__uint_as_float(o[e]), __uint_as_float(o[e + 1])), make_float2(0.f, 0.f), bad);
          if (whole) {
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
              uint4 v;
              v.x = ch_pack(__uint_as_float(o[e]) * inv, __uint_as_float(o[e + 1]) * inv);
              v.y = ch_pack(__uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv);
              v.z = ch_pack(__uint_as_float(o[e + 4]) * inv, __uint_as_float(o[e + 5]) * inv);
              v.w = ch_pack(__uint_as_float(o[e + 6]) * inv, __uint_as_float(o[e + 7]) * inv);
              if (begun) *reinterpret_cast<uint4*>(tile_at(q_buf, row, (k + e) >> 3)) = v;
              else if (place.valid) *reinterpret_cast<uint4*>((__nv_bfloat16*)p.out + out_at + k + e) = v;
            }
          } else if (place.valid) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(p.part + at * DH + k + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        tc_fence_before();
        if (whole && begun) {                  // whole rows at a time: a row per thread would write 16 bytes of 32 lines at once
          const long long mine = place.valid ? out_at : -1;
          __syncwarp();
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            const int r = i * (32 / PER) + lane / PER, ch = lane % PER;
            const long long to = __shfl_sync(0xffffffffu, mine, r);
            const uint4 v = *reinterpret_cast<const uint4*>(tile_at(q_buf, quad * 32 + r, ch));
            if (to >= 0) *reinterpret_cast<uint4*>((__nv_bfloat16*)p.out + to + ch * 8) = v;
          }
          __syncwarp();
        }
        if (place.valid) {
          if (!whole) p.part_ml[at] = make_float2(m, wild ? -1.f : l);
          else if (p.lse) p.lse[place.row * p.n_heads + place.head] = wild ? NAN : l == 0.f ? -INFINITY : fmaf(m, p.scale_log2, log2f(l)) * LN2;
        }
        if (whole && place.valid && (wild || (!(bad.x + bad.y == 0.f) && isfinite(l)))) b.redo = 1;
      }
      if constexpr (C::QBUFS == 1) {
        if (rest > 0) {
          next.next_unit(p);
          sight.learn(p, next);
          asked = ch_any(sight.of(half ^ 1, next.at, tiles_end(next, rest)));
          if (asked) {
            ask_queries(next, half ^ 1);
            hand_queries();
          }
        }
      }
      if (asked) q_buf = (uses - 1) % C::QBUFS;
      if (tid == 0) {
        if (!whole && t0 == 0) p.jobs[blockIdx.x] = make_int4(c.s, c.qt, c.head, last_worker(p, blockIdx.x, sh.piece.share, sh.piece.ahead, c.u.tiles));
        sh.piece.ahead += t1 - t0;
      }
      left = rest;
      half ^= 1;
      c = next;
    }
  }
  let_successor_start();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Nothing may land after the block is gone.  The products wait for every tile; where any warp has given up, this one does.
  if (warp == 9 && *gave_up) {
    for (int st = 0; st < C::STAGES; ++st)
      if (b.filled[st] > 0) mbar_wait_bounded(&b.full[st], (unsigned)((b.filled[st] - 1) / C::STAGES) & 1u, CH_WAIT_NS / 8);
    if (b.cleaning > 0) mbar_wait_bounded(&b.landed, (unsigned)(b.cleaning - 1), CH_WAIT_NS / 8);
  }
  if (tid == 0) p.redo[blockIdx.x] = b.redo;
  if (warp == 8) tmem_dealloc(tmem, CH_TMEM);
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
// Pages as [page][slot][head][column] (reads of more than a head's row bring in others' too soon: a step of 256 sequences of 2048,
// 16 heads of 64, took 512 us with 256 bytes at a time, 400 with 128), boxes of box_rows slots of one head, swizzled rows of box_cols (64 or 32) columns.
bool page_map(CUtensorMap* tm, const void* base, const KvView& c, int dh, int box_cols, int box_rows) {
  cuuint64_t dims[4] = {(cuuint64_t)dh, (cuuint64_t)c.n_kv, (cuuint64_t)c.page_size, (cuuint64_t)c.n_pages};
  const cuuint64_t one = (cuuint64_t)dh * 2;                       // a stride of one head or one page leads nowhere
  cuuint64_t strides[3] = {c.n_kv > 1 ? (cuuint64_t)c.ld_head * 2 : one, (cuuint64_t)c.ld_slot * 2, c.n_pages > 1 ? (cuuint64_t)c.ld_page * 2 : one};
  const cuuint32_t box[4] = {(cuuint32_t)box_cols, 1u, (cuuint32_t)box_rows, 1u};
  return encode_tensor_map(tm, 4, base, dims, strides, box, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                           dh >= 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B);
}

template <int DH>
static int launch_chunk(const AttnParams& p, cudaStream_t s) {
  int a = p.c.page_size, box = CH_TILE;
  while (a) { const int t = box % a; box = a; a = t; }
  CUtensorMap tm_k, tm_v;
  if (!page_map(&tm_k, p.c.k, p.c, DH, 64, box) || !page_map(&tm_v, p.c.v, p.c, DH, 64, box)) return PCM_ERR_CUDA;
  static std::atomic<unsigned long long> seen{0};
  if (const int rc = allow_smem(attn_chunk_kernel<DH>, ChCfg<DH>::BYTES, &seen)) return rc;
  return launch_after_smem(attn_chunk_kernel<DH>, dim3(p.workers), dim3(CH_THREADS), ChCfg<DH>::BYTES, s, tm_k, tm_v, p, box);
}
int attn_chunk_rows() { return 2 * CH_ROWS; }
int attn_chunk_tile() { return CH_TILE; }
int launch_chunk_bf16(const AttnParams& p, int dh, cudaStream_t s) { return dh == 128 ? launch_chunk<128>(p, s) : launch_chunk<64>(p, s); }

}  // namespace pga
}  // namespace pcm
