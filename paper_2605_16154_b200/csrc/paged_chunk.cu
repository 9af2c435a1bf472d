// Attention of chunks of new tokens over a paged cache in bf16, head dims 64 and 128, on the fifth-generation tensor cores.
//
// A unit is 256 rows in two streams of 128; the keys come in tiles of 128.  Per stream and tile:
//   S = Q K^T            tcgen05.mma, 128 x 128 fp32 in tensor memory
//   P = 2^(c S - c m)    four softmax warps, a thread per row: the weights are packed to bf16 over the scores they came from
//   O += P V             tcgen05.mma with P from tensor memory, accumulated there
// While one stream's warps form weights the tensor core works for the other.  The reference m of a row is its running
// maximum, but it moves only when the maximum has risen by more than 8 powers of two since: until then weights up to 2^8 are as
// exact in bf16 and fp32 as weights up to 1, and the accumulator does not have to be fetched, scaled and put back.
// Keys and values come by TMA through a ring of tiles, box by box of a page (greatest common divisor of page and tile):
// lanes of the loading warp look their boxes' pages up side by side.  Boxes that no row of the unit sees are read from
// behind the last page, which yields zeros: what the table says there does not matter.  Value rows behind the end of a sequence
// are cleared in shared memory, since a page may never have been written there.
//
// Warps 0-3 and 4-7: softmax and output of streams 0 and 1.  Warp 8: tensor memory, products.  Warp 9: loads.  Warps 10 and 11 only
// fill the warpgroup, whose registers go to the others.
// Every wait is bounded; one that expires is reported in the status word and ends the block.
#include <cuda.h>

#include "async_ptx.cuh"
#include "paged_attention.cuh"

namespace pcm {
namespace pga {

constexpr int CH_ROWS = 128, CH_TILE = 128, CH_THREADS = 384;
constexpr unsigned long long CH_WAIT_NS = 2000000000ull;
constexpr int CH_TMEM = 512;
// Registers: 168 a thread at launch, of which the last warpgroup gives up 80 so that the softmax warps, which hold a row of 128
// scores each, get 40 more: 2 x 208 + 88 = 3 x 168.
constexpr int CH_REGS_SOFTMAX = 208, CH_REGS_REST = 88;
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
constexpr float CH_RISE = 8.f;                 // powers of two by which a maximum may outgrow its reference
template <int DH> struct ChCfg {
  static constexpr int SLABS = DH / 64;        // 64 columns of 128 rows, 128-byte swizzle
  static constexpr int SLAB = 128 * 128, TILE_BYTES = SLABS * SLAB;
  static constexpr int STAGES = DH == 128 ? 5 : 10;
  static constexpr int RING_AT = 2 * TILE_BYTES, BAR_AT = RING_AT + STAGES * TILE_BYTES;
  static constexpr int BYTES = BAR_AT + 512 + 1024;                // barriers; alignment
  static constexpr int O_COL = 256;            // scores of the streams: columns 0 and 128; values: from 256 on
};

__device__ __forceinline__ void ch_load_4d(void* dst, const void* tmap, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
          smem_u32(dst)),
      "l"(tmap), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
__device__ __forceinline__ void ch_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
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
__device__ __forceinline__ void ch_tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
      "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
      "r"(r[30]), "r"(r[31])
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
    for (int i = 0; i < 32; ++i)
      if (mbar_try_wait_hint(bar, parity, 2000u)) return true;
    if (*gave_up) return false;
    if (global_timer_ns() - from > CH_WAIT_NS) {
      *gave_up = 1;
      kv_report(c, STATUS_TIMEOUT);
      return false;
    }
  }
}

// The positions of a stream's rows, and which tiles they see.
struct ChStream { int lo, hi; bool rows; };
__device__ __forceinline__ ChStream ch_stream(const AttnParams& p, const SeqSpan& sp, int qt, int s) {
  ChStream x;
  const int total = sp.fresh * p.group, r0 = qt * 2 * CH_ROWS + s * CH_ROWS;
  x.rows = r0 < total;
  const int r1 = min(total, r0 + CH_ROWS) - 1, first = sp.len - sp.fresh;
  x.lo = x.rows ? first + fast_div(r0, p.div_group) : -1;
  x.hi = x.rows ? first + fast_div(r1, p.div_group) : -1;
  return x;
}
__device__ __forceinline__ int ch_key(const UnitSpan& u, int i) { return (i < u.first_tiles ? i : i + u.skip) * CH_TILE; }
__device__ __forceinline__ bool ch_needs(const AttnParams& p, const ChStream& x, int key) {
  return x.rows && key <= x.hi && (p.window == 0 || key + CH_TILE - 1 > x.lo - p.window || key < p.sinks);
}

// Whether the stream needs one of tiles [t0, t1) of the unit.
__device__ __forceinline__ bool ch_any(const AttnParams& p, const ChStream& x, const UnitSpan& u, int t0, int t1) {
  if (x.rows)
    for (int i = t0; i < t1 && ch_key(u, i) <= x.hi; ++i)
      if (ch_needs(p, x, ch_key(u, i))) return true;
  return false;
}

struct ChBars {
  uint64_t full[10], empty[10];                // tiles of the ring
  uint64_t landed;                             // a tile that is cleaned before it is handed on
  uint64_t q_full[2], s_full[2], p_full[2], o_full[2];
  uint64_t done;
  uint32_t tmem;
  unsigned gave_up;
  int redo;
};

template <int DH>
__global__ void __launch_bounds__(CH_THREADS, 1)
attn_chunk_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ AttnParams p,
                  const int box_rows) {
  using C = ChCfg<DH>;
  extern __shared__ uint8_t ch_smem[];
  __shared__ Piece piece;
  uint8_t* base = ch_smem + ((1024u - (smem_u32(ch_smem) & 1023u)) & 1023u);
  ChBars& b = *reinterpret_cast<ChBars*>(base + C::BAR_AT);
  static_assert(sizeof(ChBars) <= 512, "barriers");
  volatile unsigned* gave_up = &b.gave_up;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < C::STAGES; ++i) { mbar_init(&b.full[i], 1); mbar_init(&b.empty[i], 1); }
    mbar_init(&b.landed, 1);
    mbar_init(&b.done, 1);
    for (int s = 0; s < 2; ++s) { mbar_init(&b.q_full[s], 4); mbar_init(&b.s_full[s], 1); mbar_init(&b.p_full[s], 4); mbar_init(&b.o_full[s], 1); }
    b.gave_up = 0;
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
  if (warp == 0) {
    Piece own;
    find_piece(p, blockIdx.x, own);
    if (lane == 0) piece = own;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = b.tmem;
  Cursor c = piece.c;
  long long left = piece.left;

  if (warp >= 8) {
    regs_down<CH_REGS_REST>();                 // the whole warpgroup at one instruction
    if (warp == 9) {
      // ---------------------------- loads ----------------------------
      // Order of the ring: K0 K1 V0 K2 V1 .., as the products want them.
      int fill = 0;                              // tiles handed to the ring so far
      unsigned landed_phase = 0;
      bool ok = true;
      const int boxes = CH_TILE / box_rows;
      auto load = [&](const Cursor& c, int i, bool values) {
        const int st = fill % C::STAGES;
        const unsigned ph = (unsigned)(fill / C::STAGES) & 1u;
        if (!ch_wait(&b.empty[st], ph ^ 1u, gave_up, p.c)) { ok = false; return; }
        uint8_t* dst = base + C::RING_AT + st * C::TILE_BYTES;
        const int key0 = ch_key(c.u, i);
        const bool clean = values && key0 + CH_TILE > c.sp.len;
        uint64_t* bar = clean ? &b.landed : &b.full[st];
        if (lane == 0) mbar_expect_tx(bar, C::TILE_BYTES);
        __syncwarp();
        if (lane < boxes * C::SLABS) {
          const int box = lane / C::SLABS, slab = lane % C::SLABS, key = key0 + box * box_rows;
          int page = p.c.n_pages, slot = 0;
          // some key of the box is seen by the unit
          const bool any = key < c.u.end && (key + box_rows > c.u.low || key < p.sinks);
          if (any) {
            const int at = fast_div(key, p.c.div_page);
            page = p.c.table[c.s * p.c.ld_table + at];
            slot = key - at * p.c.page_size;
            if (page < 0 || page >= p.c.n_pages) { page = p.c.n_pages; kv_report(p.c, STATUS_BAD_PAGE); }
          }
          ch_load_4d(dst + slab * C::SLAB + box * box_rows * 128, values ? &tm_v : &tm_k, slab * 64, c.head, slot, page, bar);
        }
        ++fill;
        if (clean) {
          __syncwarp();
          if (!ch_wait(&b.landed, landed_phase, gave_up, p.c)) { ok = false; return; }
          landed_phase ^= 1u;
          const int from = max(0, c.sp.len - key0);
          for (int r = from * C::SLABS * 8 + lane; r < CH_TILE * C::SLABS * 8; r += 32) {
            const int row = r / (C::SLABS * 8), part = r % (C::SLABS * 8);
            *reinterpret_cast<uint4*>(dst + (part >> 3) * C::SLAB + row * 128 + (part & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          ch_fence_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(&b.full[st]);
        }
      };
      while (left > 0 && ok) {
        const int t0 = c.at, t1 = (int)min((long long)c.u.tiles, t0 + left);
        load(c, t0, false);
        for (int i = t0; i < t1 && ok; ++i) {
          if (i + 1 < t1) load(c, i + 1, false);
          if (ok) load(c, i, true);
        }
        left -= t1 - t0;
        if (left > 0) c.next_unit(p);
      }
      // nothing may land after the block is gone
      for (int k = max(0, fill - C::STAGES); k < fill; ++k)
        mbar_wait_bounded(&b.full[k % C::STAGES], (unsigned)(k / C::STAGES) & 1u, CH_WAIT_NS);
    } else if (warp == 8) {
      // ---------------------------- products ----------------------------
      if (lane == 0) {
        const uint32_t q_lo = (uint32_t)ch_desc(smem_u32(base), 16u, 1024u), hi_k = (uint32_t)(ch_desc(0, 16u, 1024u) >> 32);
        const uint64_t k0 = ch_desc(smem_u32(base + C::RING_AT), 16u, 1024u), v0 = ch_desc(smem_u32(base + C::RING_AT), C::SLAB, 1024u);
        const uint32_t hi_v = (uint32_t)(v0 >> 32);
        const uint32_t idesc_s = ch_idesc(CH_TILE, 0), idesc_o = ch_idesc(DH, 1);
        auto desc = [](uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; };
        int take = 0;                            // tiles taken from the ring
        unsigned q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
        bool ok = true;
        auto scores = [&](int s, int st) {
          const uint32_t qa = q_lo + (uint32_t)(s * (C::TILE_BYTES >> 4)), ka = (uint32_t)k0 + (uint32_t)(st * (C::TILE_BYTES >> 4));
  #pragma unroll
          for (int k = 0; k < DH / 16; ++k) {
            const uint32_t o = (uint32_t)((k >> 2) * (C::SLAB >> 4) + (k & 3) * 2);
            umma_bf16(tmem + s * CH_TILE, desc(qa + o, hi_k), desc(ka + o, hi_k), idesc_s, k > 0);
          }
          umma_commit(&b.s_full[s]);
        };
        auto values = [&](int s, int st, bool first) {
          const uint32_t va = (uint32_t)v0 + (uint32_t)(st * (C::TILE_BYTES >> 4));
  #pragma unroll
          for (int k = 0; k < CH_TILE / 16; ++k)
            ch_mma_ts(tmem + C::O_COL + s * DH, tmem + s * CH_TILE + k * 8, desc(va + (uint32_t)(k * 128), hi_v), idesc_o, !(first && k == 0));
          umma_commit(&b.o_full[s]);
        };
        auto ring_wait = [&](int n) {
          if (!ch_wait(&b.full[n % C::STAGES], (unsigned)(n / C::STAGES) & 1u, gave_up, p.c)) { ok = false; return; }
          tc_fence_after();
        };
        while (left > 0 && ok) {
          const int t0 = c.at, t1 = (int)min((long long)c.u.tiles, t0 + left);
          ChStream x[2] = {ch_stream(p, c.sp, c.qt, 0), ch_stream(p, c.sp, c.qt, 1)};
          for (int s = 0; s < 2; ++s) x[s].rows = ch_any(p, x[s], c.u, t0, t1);      // a stream without tiles here brings no queries
          bool begun[2] = {false, false};
          int k_next = take;                     // ring position of the next keys
          ring_wait(k_next);
          for (int s = 0; s < 2 && ok; ++s) {
            if (!x[s].rows) continue;
            if (!ch_wait(&b.q_full[s], q_phase[s], gave_up, p.c)) { ok = false; break; }
            q_phase[s] ^= 1u;
            tc_fence_after();
            if (ch_needs(p, x[s], ch_key(c.u, t0))) scores(s, k_next % C::STAGES);
          }
          if (!ok) break;
          umma_commit(&b.empty[k_next % C::STAGES]);
          for (int i = t0; i < t1 && ok; ++i) {
            const bool more = i + 1 < t1;
            // ring: .. K(i) | K(i+1) V(i) | ..; the last V follows its K directly
            const int kn = k_next + 1, vn = more ? k_next + 2 : k_next + 1;
            bool v_here = false, k_here = false;
            for (int s = 0; s < 2 && ok; ++s) {
              if (ch_needs(p, x[s], ch_key(c.u, i))) {
                if (!ch_wait(&b.p_full[s], p_phase[s], gave_up, p.c)) { ok = false; break; }
                p_phase[s] ^= 1u;
                if (!v_here) { ring_wait(vn); v_here = true; if (!ok) break; }
                tc_fence_after();
                values(s, vn % C::STAGES, !begun[s]);
                begun[s] = true;
              }
              if (more && ch_needs(p, x[s], ch_key(c.u, i + 1))) {
                if (!k_here) { ring_wait(kn); k_here = true; if (!ok) break; }
                scores(s, kn % C::STAGES);
              }
            }
            if (!ok) break;
            if (more) {
              if (!k_here) ring_wait(kn);
              umma_commit(&b.empty[kn % C::STAGES]);
            }
            if (!v_here) ring_wait(vn);
            umma_commit(&b.empty[vn % C::STAGES]);
            k_next = more ? k_next + 2 : k_next;
            take = vn + 1;
          }
          left -= t1 - t0;
          if (left > 0) c.next_unit(p);
        }
        umma_commit(&b.done);                    // every product is over before the block frees what they use
        mbar_wait_bounded(&b.done, 0, CH_WAIT_NS);
      }
      __syncwarp();
    }
  } else {
    regs_up<CH_REGS_SOFTMAX>();
    // ---------------------------- weights and output: 128 threads a stream, a row each ----------------------------
    const int s = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t s_col = lanes + s * CH_TILE, o_col = lanes + C::O_COL + s * DH;
    uint8_t* q_smem = base + s * C::TILE_BYTES;
    unsigned s_phase = 0, o_count = 0;         // o_count: products O += P V asked for so far
    bool ok = true;
    long long ahead = piece.ahead;
    const long long share = piece.share;
    int4 job = make_int4(0, 0, 0, -1);
    // A stream's queries go to shared memory, 16 bytes a lane, as the products read them (128-byte swizzle).
    auto load_queries = [&](const Cursor& c) {
#pragma unroll 4
      for (int i = lane; i < 32 * DH / 8; i += 32) {
        const int r = quad * 32 + i / (DH / 8), ch = i % (DH / 8);
        const RowPlace x = row_place(p, c.sp, c.qt, c.head, s * CH_ROWS + r);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (x.valid) v = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)p.q + x.row * p.ld_q + x.head * p.ld_q_head + ch * 8);
        *reinterpret_cast<uint4*>(q_smem + (ch >> 3) * C::SLAB + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = v;
      }
      ch_fence_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.q_full[s]);
    };
    auto tiles_end = [&](const Cursor& c, long long left) { return (int)min((long long)c.u.tiles, c.at + left); };
    if (left > 0 && ch_any(p, ch_stream(p, c.sp, c.qt, s), c.u, c.at, tiles_end(c, left))) load_queries(c);
    while (left > 0 && ok) {
      const int t0 = c.at, t1 = (int)min((long long)c.u.tiles, t0 + left);
      const bool whole = t0 == 0 && t1 == c.u.tiles;
      const ChStream x = ch_stream(p, c.sp, c.qt, s);
      const RowPlace place = row_place(p, c.sp, c.qt, c.head, s * CH_ROWS + row);
      const int w_lo = __shfl_sync(0xffffffffu, place.pos, 0), w_hi = __reduce_max_sync(0xffffffffu, place.pos);
      float m = -INFINITY, l = 0.f;            // the row's reference, and the sum of its weights
      bool begun = false;
      for (int i = t0; i < t1; ++i) {
        const int key0 = ch_key(c.u, i);
        if (!ch_needs(p, x, key0)) continue;
        if (!ch_wait(&b.s_full[s], s_phase, gave_up, p.c)) { ok = false; break; }
        s_phase ^= 1u;
        tc_fence_after();
        uint32_t z[4][32];
#pragma unroll
        for (int k = 0; k < 4; ++k) tmem_ld_32x32(s_col + k * 32, z[k]);
        tmem_ld_wait();
        const bool all_seen = key0 + CH_TILE - 1 <= w_lo && (p.window == 0 || key0 > w_hi - p.window || key0 + CH_TILE - 1 < p.sinks);
        if (!all_seen) {
          const int last = place.pos - key0, from = p.window > 0 ? place.pos - p.window + 1 - key0 : 0, sunk = p.sinks - key0;
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const int j = k * 32 + e;
              if (j > last || (j < from && j >= sunk)) z[k][e] = __float_as_uint(-INFINITY);
            }
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float t = -INFINITY;
#pragma unroll
          for (int e = 0; e < 32; ++e) t = fmaxf(t, __uint_as_float(z[k][e]));
          top = fmaxf(top, t);
        }
        // m = -inf: nothing has been added yet but zeros, so the first maximum needs no rescaling
        const bool rise = (top - m) * p.scale_log2 > CH_RISE && m != -INFINITY;
        if (__any_sync(0xffffffffu, rise) && begun) {
          const float f = rise ? ex2((m - top) * p.scale_log2) : 1.f;
          if (!ch_wait(&b.o_full[s], (o_count - 1) & 1u, gave_up, p.c)) { ok = false; break; }
          tc_fence_after();
#pragma unroll 1
          for (int k = 0; k < DH; k += 32) {
            uint32_t o[32];
            tmem_ld_32x32(o_col + k, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            ch_tmem_st32(o_col + k, o);
          }
          ch_tmem_st_wait();
          l *= f;
        }
        if (rise || m == -INFINITY) m = top;
        const float mc = m == -INFINITY ? 0.f : -m * p.scale_log2;
        const float2 c2 = make_float2(p.scale_log2, p.scale_log2), mc2 = make_float2(mc, mc);
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float2 a = fma2(make_float2(__uint_as_float(z[k][e]), __uint_as_float(z[k][e + 1])), c2, mc2);
            a.x = ex2(a.x);
            a.y = ex2(a.y);
            sum = add2(sum, a);
            w[e >> 1] = ch_pack(a.x, a.y);
          }
          ch_tmem_st16(s_col + k * 16, w);
        }
        ch_tmem_st_wait();
        l += sum.x + sum.y;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.p_full[s]);
        ++o_count;
        begun = true;
      }
      if (!ok) break;
      // the scores of this piece are formed: the next one's queries may come in while the last values are summed
      Cursor next = c;
      const long long rest = left - (t1 - t0);
      if (rest > 0) {
        next.next_unit(p);
        if (ch_any(p, ch_stream(p, next.sp, next.qt, s), next.u, next.at, tiles_end(next, rest))) load_queries(next);
      }
      if (x.rows) {
        if (begun) {
          if (!ch_wait(&b.o_full[s], (o_count - 1) & 1u, gave_up, p.c)) { ok = false; break; }
          tc_fence_after();
        }
        const int slot = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);
        const long long at = (long long)slot * p.unit_rows + s * CH_ROWS + row;
        float* part = p.part + at * DH;
        __nv_bfloat16* out = (__nv_bfloat16*)p.out + place.row * p.ld_out + place.head * p.ld_out_head;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        float bad = 0.f;                       // NaN once a value is not finite
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
          for (int e = 0; e < 32; ++e) bad = fmaf(__uint_as_float(o[e]), 0.f, bad);
          if (place.valid) {
            if (whole) {
#pragma unroll
              for (int e = 0; e < 32; e += 8) {
                uint4 v;
                v.x = ch_pack(__uint_as_float(o[e]) * inv, __uint_as_float(o[e + 1]) * inv);
                v.y = ch_pack(__uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv);
                v.z = ch_pack(__uint_as_float(o[e + 4]) * inv, __uint_as_float(o[e + 5]) * inv);
                v.w = ch_pack(__uint_as_float(o[e + 6]) * inv, __uint_as_float(o[e + 7]) * inv);
                *reinterpret_cast<uint4*>(out + k + e) = v;
              }
            } else {
#pragma unroll
              for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(part + k + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
            }
          }
        }
        tc_fence_before();
        if (place.valid) {
          if (!whole) p.part_ml[at] = make_float2(m, l);
          else if (p.lse) p.lse[place.row * p.n_heads + place.head] = l == 0.f ? -INFINITY : fmaf(m, p.scale_log2, log2f(l)) * LN2;
        }
        if (whole && place.valid && bad != 0.f && isfinite(l)) b.redo = 1;
      }
      if (tid == 0 && !whole && t0 == 0) job = make_int4(c.s, c.qt, c.head, last_worker(p, blockIdx.x, share, ahead, c.u.tiles));
      ahead += t1 - t0;
      left = rest;
      c = next;
    }
    if (tid == 0) p.jobs[blockIdx.x] = job;
  }
  let_successor_start();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (tid == 0) p.redo[blockIdx.x] = b.redo;
  if (warp == 8) tmem_dealloc(tmem, CH_TMEM);
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeFn encode_fn() {
  static EncodeFn fn = nullptr;
  static bool tried = false;
  if (!tried) {
    tried = true;
    void* q = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &q, cudaEnableDefault, &r) == cudaSuccess && r == cudaDriverEntryPointSuccess)
      fn = (EncodeFn)q;
  }
  return fn;
}
// Pages as [page][slot][head][column], boxes of box_rows slots of one head and 64 columns.
static bool page_map(CUtensorMap* tm, const void* base, const KvView& c, int dh, int box_rows) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[4] = {(cuuint64_t)dh, (cuuint64_t)c.n_kv, (cuuint64_t)c.page_size, (cuuint64_t)c.n_pages};
  const cuuint64_t one = (cuuint64_t)dh * 2;                       // a stride of one head or one page leads nowhere
  cuuint64_t strides[3] = {c.n_kv > 1 ? (cuuint64_t)c.ld_head * 2 : one, (cuuint64_t)c.ld_slot * 2, c.n_pages > 1 ? (cuuint64_t)c.ld_page * 2 : one};
  cuuint32_t box[4] = {64u, 1u, (cuuint32_t)box_rows, 1u}, step[4] = {1, 1, 1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH>
static int launch_chunk(const AttnParams& p, cudaStream_t s) {
  int a = p.c.page_size, box = CH_TILE;
  while (a) { const int t = box % a; box = a; a = t; }
  CUtensorMap tm_k, tm_v;
  if (!page_map(&tm_k, p.c.k, p.c, DH, box) || !page_map(&tm_v, p.c.v, p.c, DH, box)) return PCM_ERR_CUDA;
  static unsigned long long seen = 0;
  if (attr_needed(&seen))
    PCM_CUDA_TRY(cudaFuncSetAttribute(attn_chunk_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, ChCfg<DH>::BYTES));
  return launch_after_smem(attn_chunk_kernel<DH>, dim3(p.workers), dim3(CH_THREADS), ChCfg<DH>::BYTES, s, tm_k, tm_v, p, box);
}
int attn_chunk_rows() { return 2 * CH_ROWS; }
int attn_chunk_tile() { return CH_TILE; }
int launch_chunk_bf16(const AttnParams& p, int dh, cudaStream_t s) { return dh == 128 ? launch_chunk<128>(p, s) : launch_chunk<64>(p, s); }

}  // namespace pga
}  // namespace pcm
