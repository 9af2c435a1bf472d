// Attention of new tokens over a paged cache: the line of work, the kernel for checks (fp32), the join of split units, and
// the entry points.  The line is described in paged_attention.cuh.
#include <cmath>

#include "async_ptx.cuh"
#include "paged_attention.cuh"

namespace pcm {
namespace pga {

// ------------------------------------------------------------------------------------------------
// tiles ahead of every sequence: one block a line
// ------------------------------------------------------------------------------------------------
constexpr int PLAN_THREADS = 1024;
// The lines of one call: few rows and many rows a sequence may each have a kernel of their own.
struct Lines { AttnParams of[2]; };
__global__ void __launch_bounds__(PLAN_THREADS) attn_plan_kernel(const __grid_constant__ Lines lines) {
  const AttnParams& p = lines.of[blockIdx.x];
  __shared__ __align__(8) unsigned char room[LINE_ROOM];
  if (p.prefix) line_prefix(p, p.prefix, room, true);
  let_successor_start();
}

// ------------------------------------------------------------------------------------------------
// fp32, few rows: 16 rows, 128 keys a tile, 16 of them for each of eight warps, which run independently of one another
// through a unit and join their sums at its end.  Bound by the latency of its loads (37 sequences of up to 701 tokens: 43 us); a
// mode for checks.
// ------------------------------------------------------------------------------------------------
constexpr int RF_ROWS = 16, RF_WARPS = 8, RF_KEYS = 16, RF_TILE = RF_WARPS * RF_KEYS, RF_THREADS = RF_WARPS * 32;
template <int DH> struct RfSmem {
  static constexpr int LDK = DH + 4;                               // a lane per key: rows shifted by a bank group
  static constexpr int WARP = RF_KEYS * LDK + RF_KEYS * DH + RF_KEYS * RF_ROWS;      // keys, values, weights
  static constexpr int FLOATS = RF_ROWS * DH + RF_WARPS * WARP + RF_WARPS * RF_ROWS * 2 + RF_ROWS * 2;
  static constexpr int BYTES = FLOATS * 4;
};

__device__ __forceinline__ void cp_async16(void* dst, const void* src, bool take) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

template <int DH>
__global__ void __launch_bounds__(RF_THREADS) attn_rows_f32_kernel(const __grid_constant__ AttnParams p) {
  using S = RfSmem<DH>;
  extern __shared__ float sm[];
  __shared__ Piece piece;
  float* qs = sm;                                                  // [16][DH]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float* ks = sm + RF_ROWS * DH + warp * S::WARP;
  float* vs = ks + RF_KEYS * S::LDK;
  float* ws = vs + RF_KEYS * DH;                                   // [key][row]
  float* all_m = sm + RF_ROWS * DH + RF_WARPS * S::WARP;           // [warp][row]
  float* all_l = all_m + RF_WARPS * RF_ROWS;
  float* row_m = all_l + RF_WARPS * RF_ROWS;                       // joined
  float* row_l = row_m + RF_ROWS;
  constexpr int CL = DH / 4, KG = 32 / CL;                         // lanes across a value's columns; keys side by side
  const int col = (lane % CL) * 4, kg = lane / CL, key_lane = lane & 15, half = lane >> 4;

  wait_for_predecessor();
  block_piece(p, sm, &piece);
  Cursor c = piece.c;
  long long left = piece.left, ahead = piece.ahead;
  const long long share = piece.share;
  int4 job = make_int4(0, 0, 0, -1);
  int redo = 0;

  while (left > 0) {
    const int t0 = c.at, t1 = (int)min((long long)c.u.tiles, t0 + left);
    const bool whole = t0 == 0 && t1 == c.u.tiles;
    for (int i = tid; i < RF_ROWS * DH; i += RF_THREADS) {
      const int r = i / DH;
      const RowPlace x = row_place(p, c.sp, c.qt, c.head, r);
      qs[i] = x.valid ? ((const float*)p.q)[x.row * p.ld_q + x.head * p.ld_q_head + (i - r * DH)] : 0.f;
    }
    int pos[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) pos[r] = row_place(p, c.sp, c.qt, c.head, half * 8 + r).pos;
    __syncthreads();
    float m[8], l[8], acc[RF_ROWS][4];
#pragma unroll
    for (int r = 0; r < 8; ++r) { m[r] = -INFINITY; l[r] = 0.f; }
#pragma unroll
    for (int r = 0; r < RF_ROWS; ++r) acc[r][0] = acc[r][1] = acc[r][2] = acc[r][3] = 0.f;
    for (int t = t0; t < t1; ++t) {
      const int key0 = (t < c.u.first_tiles ? t : t + c.u.skip) * RF_TILE + warp * RF_KEYS;
      __syncwarp();
      long long slot = -1;                     // of key key0 + lane
      if (lane < RF_KEYS && unit_sees(p, c.u, key0 + lane)) slot = slot_offset(p.c, c.s, key0 + lane, c.head);
#pragma unroll 4
      for (int i = lane; i < RF_KEYS * DH / 4; i += 32) {
        const int k = i / (DH / 4), e = (i - k * (DH / 4)) * 4;
        const long long at = __shfl_sync(0xffffffffu, slot, k);
        cp_async16(ks + k * S::LDK + e, (const float*)p.c.k + (at < 0 ? 0 : at + e), at >= 0);
        cp_async16(vs + k * DH + e, (const float*)p.c.v + (at < 0 ? 0 : at + e), at >= 0);
      }
      cp_async_wait_all();
      __syncwarp();
      float z[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) z[r] = 0.f;
      for (int e = 0; e < DH; e += 4) {
        const float4 k = *reinterpret_cast<const float4*>(ks + key_lane * S::LDK + e);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float4 q = *reinterpret_cast<const float4*>(qs + (half * 8 + r) * DH + e);
          z[r] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, z[r]))));
        }
      }
      float shrink[8];
      bool changed = false;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        if (!row_sees(p, pos[r], key0 + key_lane)) z[r] = -INFINITY;
        float top = z[r];
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float to = fmaxf(m[r], top);
        const float ref = to == -INFINITY ? 0.f : to;
        shrink[r] = m[r] == to ? 1.f : ex2((m[r] - ref) * p.scale_log2);
        changed |= shrink[r] != 1.f;
        m[r] = to;
        const float w = ex2((z[r] - ref) * p.scale_log2);
        l[r] = fmaf(l[r], shrink[r], w);
        ws[key_lane * RF_ROWS + half * 8 + r] = w;
      }
      if (__any_sync(0xffffffffu, changed)) {
#pragma unroll
        for (int r = 0; r < RF_ROWS; ++r) {
          const float f = __shfl_sync(0xffffffffu, shrink[r & 7], (r >> 3) << 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[r][i] *= f;
        }
      }
      __syncwarp();
#pragma unroll
      for (int k = kg; k < RF_KEYS; k += KG) {
        const float4 v = *reinterpret_cast<const float4*>(vs + k * DH + col);
#pragma unroll
        for (int r = 0; r < RF_ROWS; r += 4) {
          const float4 w = *reinterpret_cast<const float4*>(ws + k * RF_ROWS + r);
          acc[r][0] = fmaf(w.x, v.x, acc[r][0]); acc[r][1] = fmaf(w.x, v.y, acc[r][1]);
          acc[r][2] = fmaf(w.x, v.z, acc[r][2]); acc[r][3] = fmaf(w.x, v.w, acc[r][3]);
          acc[r + 1][0] = fmaf(w.y, v.x, acc[r + 1][0]); acc[r + 1][1] = fmaf(w.y, v.y, acc[r + 1][1]);
          acc[r + 1][2] = fmaf(w.y, v.z, acc[r + 1][2]); acc[r + 1][3] = fmaf(w.y, v.w, acc[r + 1][3]);
          acc[r + 2][0] = fmaf(w.z, v.x, acc[r + 2][0]); acc[r + 2][1] = fmaf(w.z, v.y, acc[r + 2][1]);
          acc[r + 2][2] = fmaf(w.z, v.z, acc[r + 2][2]); acc[r + 2][3] = fmaf(w.z, v.w, acc[r + 2][3]);
          acc[r + 3][0] = fmaf(w.w, v.x, acc[r + 3][0]); acc[r + 3][1] = fmaf(w.w, v.y, acc[r + 3][1]);
          acc[r + 3][2] = fmaf(w.w, v.z, acc[r + 3][2]); acc[r + 3][3] = fmaf(w.w, v.w, acc[r + 3][3]);
        }
      }
    }
    // join the warps
#pragma unroll
    for (int r = 0; r < 8; ++r) {
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
      if (key_lane == 0) { all_m[warp * RF_ROWS + half * 8 + r] = m[r]; all_l[warp * RF_ROWS + half * 8 + r] = l[r]; }
    }
#pragma unroll
    for (int r = 0; r < RF_ROWS; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = CL; d < 32; d <<= 1) acc[r][i] += __shfl_xor_sync(0xffffffffu, acc[r][i], d);
    __syncthreads();                                               // every warp is through with its keys and values
    float* mine = sm + RF_ROWS * DH + warp * S::WARP;              // [16][DH]
    if (kg == 0)
#pragma unroll
      for (int r = 0; r < RF_ROWS; ++r) *reinterpret_cast<float4*>(mine + r * DH + col) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
    __syncthreads();
    if (tid < RF_ROWS) {
      float top = -INFINITY, sum = 0.f;
      for (int w = 0; w < RF_WARPS; ++w) top = fmaxf(top, all_m[w * RF_ROWS + tid]);
      const float ref = top == -INFINITY ? 0.f : top;
      for (int w = 0; w < RF_WARPS; ++w) {
        const float f = ex2((all_m[w * RF_ROWS + tid] - ref) * p.scale_log2);
        sum = fmaf(all_l[w * RF_ROWS + tid], f, sum);
        all_m[w * RF_ROWS + tid] = f;
      }
      row_m[tid] = top; row_l[tid] = sum;
    }
    __syncthreads();
    const int slot = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);
    float* part = p.part + (long long)slot * RF_ROWS * DH;
    for (int i = tid; i < RF_ROWS * DH; i += RF_THREADS) {
      const int r = i / DH, e = i - r * DH;
      const RowPlace x = row_place(p, c.sp, c.qt, c.head, r);
      if (!x.valid) continue;
      float o = 0.f;
      for (int w = 0; w < RF_WARPS; ++w) o = fmaf(all_m[w * RF_ROWS + r], sm[RF_ROWS * DH + w * S::WARP + i], o);
      if (!whole) {
        part[i] = o;
      } else {
        ((float*)p.out)[x.row * p.ld_out + x.head * p.ld_out_head + e] = row_l[r] == 0.f ? 0.f : o / row_l[r];
        redo |= !isfinite(o) && isfinite(row_l[r]);
      }
    }
    if (tid < RF_ROWS) {
      const RowPlace x = row_place(p, c.sp, c.qt, c.head, tid);
      if (!whole) p.part_ml[(long long)slot * RF_ROWS + tid] = make_float2(row_m[tid], row_l[tid]);
      else if (x.valid && p.lse)
        p.lse[x.row * p.n_heads + x.head] = row_l[tid] == 0.f ? -INFINITY : fmaf(row_m[tid], p.scale_log2, log2f(row_l[tid])) * LN2;
    }
    __syncthreads();
    if (!whole && t0 == 0) job = make_int4(c.s, c.qt, c.head, last_worker(p, blockIdx.x, share, ahead, c.u.tiles));
    left -= t1 - t0;
    ahead += t1 - t0;
    if (left > 0) c.next_unit(p);
  }
  redo = __syncthreads_or(redo);
  if (tid == 0) { p.jobs[blockIdx.x] = job; p.redo[blockIdx.x] = redo; p.pieces[blockIdx.x] = piece; }
  let_successor_start();
}

// ------------------------------------------------------------------------------------------------
// fp32, many rows: 64 rows and a tile of 64 keys (32 at head dim 128) in registers, 8 rows by 4 (2) keys a thread: of each
// product's operands 12 vectors of four are read for 128 multiplications, so that the fp32 pipes set the pace.  The weights
// pass through shared memory between the two products; the 16 threads of 8 rows share them with nobody else.  Loads of one
// block hide behind the products of the others of its SM (4 x 1024 tokens behind 2048 to 4096, 8/4 heads of 64: 562 us, 36 TFLOP/s).
// ------------------------------------------------------------------------------------------------
constexpr int TF_ROWS = 64, TF_THREADS = 128;
template <int DH> struct TfCfg {
  static constexpr int KEYS = DH == 128 ? 32 : 64, KT = KEYS / 16;                 // keys of a tile, of a thread
  static constexpr int LDQ = DH + 4, LDP = KEYS + 4;               // eight rows of a vector never share banks
  static constexpr int COLS = DH / 16, VEC = COLS < 4 ? COLS : 4;  // columns of a thread, in vectors
  static constexpr int FLOATS = TF_ROWS * LDQ + KEYS * LDQ + KEYS * DH + TF_ROWS * LDP;
  static constexpr int BYTES = FLOATS * 4;
};

template <int DH>
__global__ void __launch_bounds__(TF_THREADS) attn_tiles_f32_kernel(const __grid_constant__ AttnParams p) {
  using C = TfCfg<DH>;
  extern __shared__ float sm[];
  __shared__ Piece piece;
  __shared__ long long slots[2][C::KEYS];
  float* qs = sm;
  float* ks = qs + TF_ROWS * C::LDQ;
  float* vs = ks + C::KEYS * C::LDQ;
  float* ps = vs + C::KEYS * DH;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;

  wait_for_predecessor();
  block_piece(p, sm, &piece);
  Cursor c = piece.c;
  long long left = piece.left, ahead = piece.ahead;
  const long long share = piece.share;
  int4 job = make_int4(0, 0, 0, -1);
  int redo = 0;

  while (left > 0) {
    const int t0 = c.at, t1 = (int)min((long long)c.u.tiles, t0 + left);
    const bool whole = t0 == 0 && t1 == c.u.tiles;
    auto first_key = [&](int t) { return (t < c.u.first_tiles ? t : t + c.u.skip) * C::KEYS; };
    auto look_up = [&](int t) {                // where the keys of tile t lie
      if (tid < C::KEYS) {
        const int key = first_key(t) + tid;
        slots[t & 1][tid] = unit_sees(p, c.u, key) ? slot_offset(p.c, c.s, key, c.head) : -1;
      }
    };
    for (int i = tid; i < TF_ROWS * DH / 4; i += TF_THREADS) {
      const int r = i / (DH / 4), e = (i - r * (DH / 4)) * 4;
      const RowPlace x = row_place(p, c.sp, c.qt, c.head, r);
      float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
      if (x.valid) q = *reinterpret_cast<const float4*>((const float*)p.q + x.row * p.ld_q + x.head * p.ld_q_head + e);
      *reinterpret_cast<float4*>(qs + r * C::LDQ + e) = q;
    }
    int pos[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pos[i] = row_place(p, c.sp, c.qt, c.head, ty * 8 + i).pos;
    float m[8], l[8], o[8][C::COLS];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int j = 0; j < C::COLS; ++j) o[i][j] = 0.f;
    }
    look_up(t0);
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
      const int key0 = first_key(t);
#pragma unroll 4
      for (int i = tid; i < C::KEYS * DH / 4; i += TF_THREADS) {
        const int k = i / (DH / 4), e = (i - k * (DH / 4)) * 4;
        const long long at = slots[t & 1][k];
        cp_async16(ks + k * C::LDQ + e, (const float*)p.c.k + (at < 0 ? 0 : at + e), at >= 0);
        cp_async16(vs + k * DH + e, (const float*)p.c.v + (at < 0 ? 0 : at + e), at >= 0);
      }
      if (t + 1 < t1) look_up(t + 1);
      cp_async_wait_all();
      __syncthreads();
      float z[8][C::KT];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < C::KT; ++j) z[i][j] = 0.f;
#pragma unroll 2
      for (int e = 0; e < DH; e += 4) {
        float4 k[C::KT];
#pragma unroll
        for (int j = 0; j < C::KT; ++j) k[j] = *reinterpret_cast<const float4*>(ks + (tx + 16 * j) * C::LDQ + e);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float4 q = *reinterpret_cast<const float4*>(qs + (ty * 8 + i) * C::LDQ + e);
#pragma unroll
          for (int j = 0; j < C::KT; ++j) z[i][j] = fmaf(q.x, k[j].x, fmaf(q.y, k[j].y, fmaf(q.z, k[j].z, fmaf(q.w, k[j].w, z[i][j]))));
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < C::KT; ++j) {
          if (!row_sees(p, pos[i], key0 + tx + 16 * j)) z[i][j] = -INFINITY;
          top = fmaxf(top, z[i][j]);
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        if (top > m[i]) {
          const float f = ex2((m[i] - top) * p.scale_log2);
          m[i] = top;
          l[i] *= f;
#pragma unroll
          for (int j = 0; j < C::COLS; ++j) o[i][j] *= f;
        }
        const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
        for (int j = 0; j < C::KT; ++j) {
          const float w = ex2((z[i][j] - ref) * p.scale_log2);
          l[i] += w;
          ps[(ty * 8 + i) * C::LDP + tx + 16 * j] = w;
        }
      }
      __syncwarp();
#pragma unroll 2
      for (int k = 0; k < C::KEYS; k += 4) {
        float v[4][C::COLS];
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int j = 0; j < C::COLS; j += C::VEC) {
            const float* from = vs + (k + n) * DH + j * 16 + tx * C::VEC;
            if (C::VEC == 4) *reinterpret_cast<float4*>(&v[n][j]) = *reinterpret_cast<const float4*>(from);
            else *reinterpret_cast<float2*>(&v[n][j]) = *reinterpret_cast<const float2*>(from);
          }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float4 w = *reinterpret_cast<const float4*>(ps + (ty * 8 + i) * C::LDP + k);
#pragma unroll
          for (int j = 0; j < C::COLS; ++j) o[i][j] = fmaf(w.x, v[0][j], fmaf(w.y, v[1][j], fmaf(w.z, v[2][j], fmaf(w.w, v[3][j], o[i][j]))));
        }
      }
      __syncthreads();                         // the next tile's keys and values take the place of these
    }
    const int slot = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
      const int r = ty * 8 + i;
      const RowPlace x = row_place(p, c.sp, c.qt, c.head, r);
      if (!x.valid) continue;
      const long long at = (long long)slot * TF_ROWS + r;
      float* to = whole ? (float*)p.out + x.row * p.ld_out + x.head * p.ld_out_head : p.part + at * DH;
      const float by = !whole ? 1.f : l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
      for (int j = 0; j < C::COLS; ++j) {
        redo |= whole && !isfinite(o[i][j]) && isfinite(l[i]);
        to[(j / C::VEC) * C::VEC * 16 + tx * C::VEC + j % C::VEC] = o[i][j] * by;
      }
      if (tx == 0) {
        if (!whole) p.part_ml[at] = make_float2(m[i], l[i]);
        else if (p.lse) p.lse[x.row * p.n_heads + x.head] = l[i] == 0.f ? -INFINITY : fmaf(m[i], p.scale_log2, log2f(l[i])) * LN2;
      }
    }
    if (!whole && t0 == 0) job = make_int4(c.s, c.qt, c.head, last_worker(p, blockIdx.x, share, ahead, c.u.tiles));
    left -= t1 - t0;
    ahead += t1 - t0;
    if (left > 0) c.next_unit(p);
  }
  redo = __syncthreads_or(redo);
  if (tid == 0) { p.jobs[blockIdx.x] = job; p.redo[blockIdx.x] = redo; p.pieces[blockIdx.x] = piece; }
  let_successor_start();
}

// ------------------------------------------------------------------------------------------------
// join of split units: a warp per row, the pieces in the order of their keys; and rows formed once more
// ------------------------------------------------------------------------------------------------
constexpr int JN_WARPS = 8, JN_BLOCKS = 8;     // warps a block; blocks for a worker's rows: one wave of them for 148 workers

template <typename T, int DH>
__device__ void store_row(const AttnParams& p, const RowPlace& x, const float (&o)[DH / 32]) {
  T* out = (T*)p.out + x.row * p.ld_out + x.head * p.ld_out_head + (threadIdx.x & 31);
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) from_float(out[32 * i], o[i]);
}

// Row r of the whole units of worker w, where it is not finite.
template <typename T, int DH>
__device__ __noinline__ void redo_rows(const AttnParams& p, int w, int r) {
  Piece piece = p.pieces[w];
  Cursor& c = piece.c;
  while (piece.left > 0) {
    const RowPlace x = row_place(p, c.sp, c.qt, c.head, r);
    if (c.at == 0 && c.u.tiles <= piece.left && x.valid) {
      const T* out = (const T*)p.out + x.row * p.ld_out + x.head * p.ld_out_head + (threadIdx.x & 31);
      bool fine = true;
      for (int i = 0; i < DH; i += 32) fine &= (bool)isfinite(as_float(out[i]));
      if (__any_sync(0xffffffffu, !fine)) {
        float o[DH / 32];
        const float lse = exact_row<T, DH>(p, c.s, c.head, c.u, x, o);
        store_row<T, DH>(p, x, o);
        if (p.lse && (threadIdx.x & 31) == 0) {
          float& kept = p.lse[x.row * p.n_heads + x.head];
          if (kept != kept) kept = lse;        // NaN: the row's weights did not fit either
        }
      }
    }
    piece.left -= min((long long)c.u.tiles - c.at, piece.left);
    if (piece.left > 0) c.next_unit(p);
  }
}

template <typename T, int DH>
__global__ void __launch_bounds__(JN_WARPS * 32) attn_join_kernel(const __grid_constant__ Lines lines) {
  const AttnParams& p = lines.of[blockIdx.z];
  const int w0 = blockIdx.x, r0 = blockIdx.y * JN_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  wait_for_predecessor();
  if (w0 >= p.workers) return;
  const int4 job = p.jobs[w0];
  if (p.redo[w0])
    for (int r = r0; r < p.unit_rows; r += gridDim.y * JN_WARPS) redo_rows<T, DH>(p, w0, r);
  if (job.w < 0) return;
  const SeqSpan sp = attn_span(p, job.x, false);
  const int n = job.w - w0 + 1;                // pieces: the second of worker w0, the first ones of those behind it
  constexpr int C = DH / 32;
  for (int r = r0; r < p.unit_rows; r += gridDim.y * JN_WARPS) {
    const RowPlace x = row_place(p, sp, job.y, job.z, r);
    if (!x.valid) return;
    auto place_of = [&](int i) { return (long long)(i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)) * p.unit_rows + r; };
    float v[4][C];                             // four pieces' values, on their way before their weights are known
    auto fetch = [&](int i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* part = p.part + place_of(i + j) * DH + lane;
#pragma unroll
        for (int k = 0; k < C; ++k) v[j][k] = i + j < n ? part[32 * k] : 0.f;
      }
    };
    float2 first = make_float2(-INFINITY, 0.f);
    if (lane < n) first = p.part_ml[place_of(lane)];
    fetch(0);
    float top = first.x;
    for (int i = lane + 32; i < n; i += 32) top = fmaxf(top, p.part_ml[place_of(i)].x);
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
    const float ref = top == -INFINITY ? 0.f : top;
    float o[C], l = 0.f;
    bool unfit = false;
#pragma unroll
    for (int k = 0; k < C; ++k) o[k] = 0.f;
    for (int base = 0; base < n; base += 32) {                     // a lane per piece, then the pieces in order
      float2 ml = base == 0 ? first : make_float2(-INFINITY, 0.f);
      if (base > 0 && base + lane < n) ml = p.part_ml[place_of(base + lane)];
      const float f = ex2((ml.x - ref) * p.scale_log2);
      l = fmaf(ml.y, f, l);
      unfit |= ml.y < 0.f;                     // a piece whose weights did not fit
      const int here = min(32, n - base);
      for (int i = 0; i < here; i += 4) {
        if (base + i > 0) fetch(base + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float g = __shfl_sync(0xffffffffu, f, (i + j) & 31);
          if (i + j < here)
#pragma unroll
            for (int k = 0; k < C; ++k) o[k] = fmaf(v[j][k], g, o[k]);
        }
      }
    }
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) l += __shfl_xor_sync(0xffffffffu, l, k);
    unfit = __any_sync(0xffffffffu, unfit);
    bool fine = true;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      fine &= (bool)isfinite(o[k]);
      o[k] = l == 0.f ? 0.f : o[k] / l;
    }
    float lse = l == 0.f ? -INFINITY : fmaf(top, p.scale_log2, log2f(l)) * LN2;
    if (unfit || (__any_sync(0xffffffffu, !fine) && isfinite(l))) {
      const float exact = exact_row<T, DH>(p, job.x, job.z, unit_span(p, sp, job.y), x, o);
      if (unfit) lse = exact;
    }
    store_row<T, DH>(p, x, o);
    if (lane == 0 && p.lse) p.lse[x.row * p.n_heads + x.head] = lse;
  }
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
template <int DH>
static int launch_f32(const AttnParams& p, cudaStream_t s) {
  static std::atomic<unsigned long long> seen{0};
  if (const int rc = allow_smem(attn_rows_f32_kernel<DH>, RfSmem<DH>::BYTES, &seen)) return rc;
  return launch_after_smem(attn_rows_f32_kernel<DH>, dim3(p.workers), dim3(RF_THREADS), RfSmem<DH>::BYTES, s, p);
}

template <int DH>
static int launch_tiles_f32(const AttnParams& p, cudaStream_t s) {
  static std::atomic<unsigned long long> seen{0};
  if (const int rc = allow_smem(attn_tiles_f32_kernel<DH>, TfCfg<DH>::BYTES, &seen)) return rc;
  return launch_after_smem(attn_tiles_f32_kernel<DH>, dim3(p.workers), dim3(TF_THREADS), TfCfg<DH>::BYTES, s, p);
}

template <typename T, int DH>
static int launch_join(const Lines& a, int n, cudaStream_t s) {
  int workers = 0, rows = 0;
  for (int i = 0; i < n; ++i) { workers = max(workers, a.of[i].workers); rows = max(rows, a.of[i].unit_rows); }
  return launch_after(attn_join_kernel<T, DH>, dim3(workers, min(JN_BLOCKS, ceil_div(rows, JN_WARPS)), n), dim3(JN_WARPS * 32), s, a);
}
template <typename T>
static int launch_join_as(const Lines& a, int n, int dh, cudaStream_t s) {
  return dh == 128 ? launch_join<T, 128>(a, n, s) : dh == 64 ? launch_join<T, 64>(a, n, s) : launch_join<T, 32>(a, n, s);
}

struct Layout { size_t prefix, jobs, redo, pieces, ml, part, total; };
static Layout layout(int n_seq, int workers, int unit_rows, int dh) {
  Layout y;
  auto up = [](size_t b) { return (b + 255) / 256 * 256; };
  y.prefix = 0;
  y.jobs = y.prefix + up(((size_t)n_seq + 1) * 8);
  y.redo = y.jobs + up((size_t)workers * 16);
  y.pieces = y.redo + up((size_t)workers * 4);
  y.ml = y.pieces + up((size_t)workers * sizeof(Piece));
  y.part = y.ml + up((size_t)2 * workers * unit_rows * 8);
  y.total = y.part + up((size_t)2 * workers * unit_rows * dh * 4);
  return y;
}
static void place(AttnParams& p, const Layout& y, void* ws) {
  unsigned char* b = (unsigned char*)ws;
  p.prefix = (long long*)(b + y.prefix);
  p.jobs = (int4*)(b + y.jobs);
  p.redo = (int*)(b + y.redo);
  p.pieces = (Piece*)(b + y.pieces);
  p.part_ml = (float2*)(b + y.ml);
  p.part = (float*)(b + y.part);
}

static bool attn_sizes_ok(const grpo_kv_cache* c, int64_t n_seq, int64_t n_rows, int64_t n_heads) {
  if (!c || (c->dtype != GRPO_F32 && c->dtype != GRPO_BF16) || n_seq < 0 || n_rows < 0 || c->n_kv_heads < 1 || n_heads < 1) return false;
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return false;
  if (n_heads % c->n_kv_heads || n_heads > (1 << 16) || n_seq > PCM_MAX_VOCAB_CALL || n_rows > PCM_MAX_VOCAB_CALL) return false;
  return n_rows * (n_heads / c->n_kv_heads) <= PCM_MAX_VOCAB_CALL;              // rows of a key-value head are counted in 32 bits
}

// Rows of a key-value head (new tokens times group) up to which a sequence goes to the kernel for few rows; one head each below.
// bf16, two row tiles at head dim 64 (300, 2000 and 8000 tokens of 256, 40 and 16 sequences, 32 rows: 89, 38 and 50 us, 104, 46 and 61
// in the kernel for many; 48 rows: 149, 57 and 75 against 110, 48 and 63), one at 128, whose registers hold no more (16 rows: 94, 46
// and 63 us against 124, 55 and 68; 24 rows: 161, 69 and 89 against 124, 55 and 67).  Head dim 32 has the one kernel.
// fp32: where sequences of few and of many rows meet, a border of 16 takes a launch of either kernel after the other (37 sequences of
// up to 120 rows: 41 us, 72 with it); batches of one size between 17 and 128 rows would be better off with it (40 sequences of 300
// tokens, 32 rows of head dim 64: 61 us, 51; 128 rows: 159, 79).
static int few_rows_of(int dtype, int dh) { return dtype == GRPO_F32 ? 128 : dh == 128 ? 16 : 32; }

// The lines of a call: which kernels take part, with what workers; n_lines and their regions of the workspace.
struct CallPlan { int n; bool planned, self[2], chunk[2]; int rows[2], tile[2], workers[2], min_share[2], over[2], up_to[2]; Layout at[2]; size_t total; };
static CallPlan plan_call(int dtype, int dh, int n_seq, int n_rows, int group, int max_new) {
  CallPlan c;
  c.n = 0; c.total = 0; c.planned = false;
  const long long new_most = max_new > 0 && max_new < n_rows ? max_new : n_rows, most = new_most * group;
  auto add = [&](bool chunk, int rows, int tile, int workers, int min_share, int over, int up_to) {
    const int i = c.n++;
    c.chunk[i] = chunk; c.rows[i] = rows; c.tile[i] = tile; c.workers[i] = workers; c.min_share[i] = min_share;
    c.over[i] = over; c.up_to[i] = up_to;
    c.at[i] = layout(n_seq, workers, rows, dh);
    c.total += c.at[i].total;
    // most row tiles that the call's rows can make
    c.self[i] = n_seq <= SELF_PLANNED && (long long)n_rows * group / rows + n_seq <= SELF_PLANNED;
    c.planned |= !c.self[i];
  };
  const int all = 0x7FFFFFFF, sms = sm_count();
  // sequences of many rows have a kernel of their own, and so do those of few; where every sequence brings max_new rows, none has few
  const bool f32 = dtype == GRPO_F32;
  const int few_rows = few_rows_of(dtype, dh);
  const bool many = most > few_rows && (f32 || dh != 32), few = !many || (long long)n_seq * new_most != n_rows;
  if (few && f32) add(false, RF_ROWS, RF_TILE, 2 * sms, 4, 0, many ? few_rows : all);
  if (few && !f32) add(false, most <= 16 || few_rows == 16 ? 16 : 32, attn_rows_tile(dh), 2 * sms, 1, 0, many ? few_rows : all);
  if (many && f32) add(true, TF_ROWS, dh == 128 ? TfCfg<128>::KEYS : TfCfg<64>::KEYS, (dh == 128 ? 2 : 3) * sms, 1, few ? few_rows : 0, all);
  if (many && !f32) add(true, attn_chunk_rows(), attn_chunk_tile(), sms, 4, few ? few_rows : 0, all);
  return c;
}

// A wait for a barrier that nothing arrives at, reported as the kernels above report theirs.
__global__ void expired_wait_kernel(KvView c) {
  __shared__ uint64_t never;
  mbar_init(&never, 1);
  fence_mbar_init();
  if (!mbar_wait_bounded(&never, 0, 1000000ull)) kv_report_expired(c);
}

}  // namespace pga
}  // namespace pcm

using namespace pcm;
using namespace pcm::pga;

extern "C" size_t grpo_paged_attention_workspace_bytes(const grpo_kv_cache* cache, int32_t n_seq, int32_t n_rows, int32_t n_heads,
                                                       int32_t max_new) {
  if (!attn_sizes_ok(cache, n_seq, n_rows, n_heads) || max_new < 0) return 0;
  // as large as any smaller call's: few rows alone, or few and many
  const int group = n_heads / cache->n_kv_heads;
  const CallPlan c = plan_call(cache->dtype, cache->head_dim, n_seq, n_rows, group, max_new);
  size_t total = layout(n_seq, 2 * sm_count(), cache->dtype == GRPO_F32 ? RF_ROWS : 32, cache->head_dim).total;
  if (c.chunk[c.n - 1]) total += c.at[c.n - 1].total;
  return total;
}

extern "C" int grpo_paged_attention(const grpo_kv_cache* cache, const grpo_kv_batch* batch, int32_t n_rows, const void* q, int64_t ld_q,
                                    int64_t ld_q_head, int32_t n_heads, float scale, int32_t window, int32_t sinks, int32_t max_new,
                                    void* out, int64_t ld_out, int64_t ld_out_head, float* lse, uint32_t* device_status, void* workspace,
                                    size_t workspace_bytes, pcm_stream stream) {
  const int bad = kv_check(cache, batch, n_rows);
  if (bad != PCM_OK) return bad;
  if (n_heads < 1 || !(scale > 0.f) || !std::isfinite(scale * LOG2E) || window < 0 || sinks < 0 || max_new < 0) return PCM_ERR_ARG;
  if (n_heads % cache->n_kv_heads) return PCM_ERR_ARG;
  if (!attn_sizes_ok(cache, batch->n_seq, n_rows, n_heads)) return PCM_ERR_SHAPE;
  if (n_rows == 0 || batch->n_seq == 0) return PCM_OK;
  const int dh = cache->head_dim;
  if (!q || !out || (lse && ((uintptr_t)lse & 3))) return PCM_ERR_ARG;
  if ((n_heads > 1 && ld_q_head < dh) || (n_rows > 1 && ld_q < dh) || rows_overlap(n_rows, n_heads, dh, ld_out, ld_out_head)) return PCM_ERR_ARG;
  const int64_t per = cache->dtype == GRPO_BF16 ? 8 : 4;
  if ((((uintptr_t)q | (uintptr_t)out) & 15) || (n_heads > 1 && (ld_q_head % per || ld_out_head % per)) ||
      (n_rows > 1 && (ld_q % per || ld_out % per)))
    return PCM_ERR_SHAPE;
  if (!workspace || ((uintptr_t)workspace & 255) ||
      workspace_bytes < grpo_paged_attention_workspace_bytes(cache, batch->n_seq, n_rows, n_heads, max_new))
    return PCM_ERR_WORKSPACE;
  AttnParams p = {};
  p.c = kv_view(cache, batch, n_rows, device_status);
  if (!p.c.waits && !(p.c.waits = tcgen05_status_word())) return PCM_ERR_CUDA;      // (left for the next call that polls)
  p.q = q; p.ld_q = n_rows > 1 ? ld_q : 0; p.ld_q_head = n_heads > 1 ? ld_q_head : 0;
  p.out = out; p.ld_out = n_rows > 1 ? ld_out : 0; p.ld_out_head = n_heads > 1 ? ld_out_head : 0;
  p.lse = lse;
  p.n_heads = n_heads; p.group = n_heads / cache->n_kv_heads;
  p.div_group = make_fastdiv(p.group);
  p.scale_log2 = scale * LOG2E;
  p.window = window; p.sinks = sinks < PCM_MAX_VOCAB_CALL ? sinks : PCM_MAX_VOCAB_CALL;       // (no sequence is longer: sums with tiles fit)
  cudaStream_t s = (cudaStream_t)stream;
  prof_begin(PC_ATTN, s);
  const bool bf16 = cache->dtype == GRPO_BF16;
  const CallPlan call = plan_call(cache->dtype, dh, batch->n_seq, n_rows, p.group, batch->q_off ? max_new : 1);
  Lines lines;
  unsigned char* ws = (unsigned char*)workspace;
  for (int i = 0; i < call.n; ++i) {
    AttnParams& a = lines.of[i];
    a = p;
    a.unit_rows = call.rows[i]; a.tile = call.tile[i]; a.tile_shift = __builtin_ctz(call.tile[i]); a.row_shift = __builtin_ctz(call.rows[i]); a.workers = call.workers[i]; a.min_share = call.min_share[i];
    a.over_rows = call.over[i]; a.up_to_rows = call.up_to[i];
    place(a, call.at[i], ws);
    if (call.self[i]) a.prefix = nullptr;
    ws += call.at[i].total;
  }
  int rc = PCM_OK;
  if (call.planned) {
    attn_plan_kernel<<<call.n, PLAN_THREADS, 0, s>>>(lines);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); rc = PCM_ERR_CUDA; }
  }
  for (int i = 0; i < call.n && rc == PCM_OK; ++i) {
    const AttnParams& a = lines.of[i];
    if (!bf16 && call.chunk[i]) rc = dh == 128 ? launch_tiles_f32<128>(a, s) : dh == 64 ? launch_tiles_f32<64>(a, s) : launch_tiles_f32<32>(a, s);
    else if (!bf16) rc = dh == 128 ? launch_f32<128>(a, s) : dh == 64 ? launch_f32<64>(a, s) : launch_f32<32>(a, s);
    else rc = call.chunk[i] ? launch_chunk_bf16(a, dh, s) : launch_rows_bf16(a, dh, s);
  }
  if (rc == PCM_OK) rc = bf16 ? launch_join_as<__nv_bfloat16>(lines, call.n, dh, s) : launch_join_as<float>(lines, call.n, dh, s);
  prof_end(s, 0.0, 0.0);                       // (bytes and products follow from lengths that only the device knows)
  return rc;
}

extern "C" int grpo_expired_wait(uint32_t* device_status, pcm_stream stream) {
  if ((uintptr_t)device_status & 3) return PCM_ERR_ARG;
  KvView c = {};
  c.waits = device_status ? device_status : tcgen05_status_word();
  if (!c.waits) return PCM_ERR_CUDA;
  expired_wait_kernel<<<1, 1, 0, (cudaStream_t)stream>>>(c);
  PCM_LAUNCH_CHECK();
  return PCM_OK;
}
