// Log-probabilities of given tokens straight from the last hidden states x [M][d] and the head's weight w [V][d], and
// their gradients.  The logits z = x w^T exist only as accumulator tiles in tensor memory:
//   forward   the head GEMM's epilogue reduces each half tile of a row to softmax statistics (16 bytes instead of the
//             256 or 512 of up to 128 logits); a small kernel joins them.  Bound by the tensor cores from a few
//             hundred rows on, by reading w below.
//   backward  the same product once more, its epilogue writing d loss / d z in bf16 (rounded value and remainder) for a
//             chunk of rows; then dx = dz w and dw (+)= dz^T x.
// Both are bound by the tensor cores under the board's power limit.  21504 rows x 1024 x 32000: forward 0.98 ms in calls back
// to back and 1.15 ms on inputs that change from call to call (1430 and 1225 TFLOP/s), backward 4.5 and 5.35 ms; 16 rows x 2048 x
// 32000 forward: 28 - 30 us, of which w (131 MB) takes 20.
// Roundings to fewer bits: d z enters dx in bf16, the target's entry corrected by what that leaves (corr w[tok], added before
// dx is rounded).  The rounding of the result itself is 1.66e-3 of dx's norm.  Where the policy is flat (logits of spread 1.5)
// the target carries d z and the error stays there; where another token carries as much, its rounding shows: 1.8e-3 at spread 4,
// 1.9 - 2.05e-3 at 8 to 20 (701 x 1024 x 5003; worst row 3.1e-3, of a rounded exact result 1.8e-3).  GRPO_EXACT_DX takes
// d z as hi + lo here too: 1.66e-3 everywhere, for a fifth product (21504 x 1024 x 32000: 6.3 ms instead of 4.5 back to back,
// 6.65 instead of 5.35 on changing inputs; 701 x 1024 x 5003: 98 us instead of 93).
// dw is fp32, so its d z enters as hi + lo, two bf16 values, 16 significant bits, and the
// target's d z, mostly the largest of its row, apart: coef x summed by token in fp32 (embed_accumulate_sum).  Relative to
// dw's norm that leaves 0.8e-6 (701 rows x 1024 x 5003) and 0.35e-6 (8192 x 1024 x 32000), where fp32 products leave 0.5e-6
// and 1.6e-6; hi + lo alone left 2.6e-6, hi alone would leave 1.6e-3.  The sums cost 60 us of the large batch, 19 us of
// 86 of the small one.

#include "internal.h"

namespace pcm {

constexpr int VH_GROUPS = 16;                 // column-block slices of a row joined side by side
// k-blocks (of 64 rows) per accumulator piece of dw.  8192 rows x 1024 x 32000: error 2.55e-6 / 2.60e-6 / 2.81e-6 with 4 / 8 /
// 16 (before the targets went apart), time the same within the clock's wandering; without pieces the drift grows with the rows (4e-5 at 119808).
constexpr int VH_CHAIN_KB = 8;

struct JoinParams {
  const float4* part;                         // [parts][M]
  int M, V, bn, parts;                        // columns per tile; two parts a tile
  const int* tok;
  float inv_t;
  float* logp; float* entropy; float* lse;
  unsigned* status;
};

__device__ __forceinline__ VocabStat load_part(const JoinParams& p, int b, long long row) {
  const float4 q = p.part[(long long)b * p.M + row];
  return VocabStat{q.x, q.y, q.z};
}
__device__ __forceinline__ void finish_row(const JoinParams& p, const VocabStat& st, long long row) {
  const int t = p.tok[row];
  const bool live = t >= 0 && t < p.V;
  if (t >= p.V && p.status) atomicOr(p.status, STATUS_BAD_TOKEN);
  const RowResult res(st, p.inv_t);
  if (p.logp) p.logp[row] = live ? res.logp(p.part[(long long)(2 * (t / p.bn) + (t % p.bn) / 128) * p.M + row].w) : 0.f;
  if (p.entropy) p.entropy[row] = live ? res.entropy : 0.f;
  if (p.lse) p.lse[row] = live ? res.lse : 0.f;
}

// Many rows: 32 per block; thread (lane, slice) runs over every 16th part of row 32 b + lane (a warp reads 512 contiguous
// bytes), then slice 0 joins the slices.
__global__ void __launch_bounds__(32 * VH_GROUPS)
vocab_stats_join_kernel(const JoinParams p) {
  __shared__ VocabStat sm[VH_GROUPS][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const long long row = (long long)blockIdx.x * 32 + lane;
  const float c = p.inv_t * VOCAB_LOG2E;
  wait_for_predecessor();
  VocabStat st{-INFINITY, 0.f, 0.f};
  if (row < p.M) {
#pragma unroll 4
    for (int b = slice; b < p.parts; b += VH_GROUPS) st = stat_join(st, load_part(p, b, row), c);
  }
  sm[slice][lane] = st;
  __syncthreads();
  if (slice != 0 || row >= p.M) return;
  for (int k = 1; k < VH_GROUPS; ++k) st = stat_join(st, sm[k][lane], c);
  finish_row(p, st, row);
}

// Few rows: one per block, so that a row's parts are read at once.
__global__ void __launch_bounds__(128)
vocab_stats_join_row_kernel(const JoinParams p) {
  __shared__ VocabStat sm[4];
  const int tid = threadIdx.x;
  const float c = p.inv_t * VOCAB_LOG2E;
  wait_for_predecessor();
  VocabStat st{-INFINITY, 0.f, 0.f};
#pragma unroll 4
  for (int b = tid; b < p.parts; b += 128) st = stat_join(st, load_part(p, b, blockIdx.x), c);
#pragma unroll
  for (int off = 16; off; off >>= 1) {
    VocabStat o;
    o.m = __shfl_down_sync(0xffffffffu, st.m, off);
    o.s = __shfl_down_sync(0xffffffffu, st.s, off);
    o.w = __shfl_down_sync(0xffffffffu, st.w, off);
    st = stat_join(st, o, c);
  }
  if ((tid & 31) == 0) sm[tid >> 5] = st;
  __syncthreads();
  if (tid != 0) return;
  for (int k = 1; k < 4; ++k) st = stat_join(st, sm[k], c);
  finish_row(p, st, blockIdx.x);
}

// The hidden states with zeros in the rows that have no token (or no finite logit, lse = -inf): their d z is zero, but zero
// times whatever such a row holds (NaN, inf) need not be.
__global__ void __launch_bounds__(256)
live_rows_kernel(const uint4* __restrict__ x, long long ld8, int M, int d8, const int* __restrict__ tok,
                 const float* __restrict__ lse, int V, uint4* __restrict__ out, unsigned* status, int beside) {
  // `beside`: launched behind the sort of the chunk's tokens, which began when all before it had ended, so that the rows
  // can be copied while it runs; this kernel ends when both are done.  Otherwise the chunk before may still be read.
  if (!beside) wait_for_predecessor();
  let_successor_start();
  const long long total = (long long)M * d8;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long row = i / d8;
    const int c = (int)(i - row * d8), t = tok[row];
    const bool live = t >= 0 && t < V && lse[row] != -INFINITY;
    if (t >= V && c == 0 && status) atomicOr(status, STATUS_BAD_TOKEN);
    out[i] = live ? x[row * ld8 + c] : make_uint4(0, 0, 0, 0);
  }
  if (beside) wait_for_predecessor();
}

// Parts of a split contraction added in order, four columns a thread.
template <bool BF16>
__global__ void __launch_bounds__(256)
parts_sum_kernel(const float* __restrict__ part, long long stride, int splits, long long M, int N, void* __restrict__ C, long long ldc,
                 int accumulate, const VocabHeadArgs vh) {
  wait_for_predecessor();
  let_successor_start();
  const int n4 = N / 4;
  const long long total = M * n4;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long row = i / n4;
    const int col = (int)(i - row * n4) * 4;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int k = 0; k < splits; ++k) {
      const float4 w = __ldcs(reinterpret_cast<const float4*>(part + (long long)k * stride + row * N + col));
      a.x += w.x; a.y += w.y; a.z += w.z; a.w += w.w;
    }
    if constexpr (BF16) {
      const int t = vh.corr ? vh.tok[row] : -1;                     // as in the product's own epilogue
      if (t >= 0 && t < vh.vocab) {
        const uint2 q = __ldg(reinterpret_cast<const uint2*>(vh.w + (long long)t * vh.ld_w + col));
        const float k = vh.corr[row];
        a.x += k * __uint_as_float(q.x << 16); a.y += k * __uint_as_float(q.x & 0xFFFF0000u);
        a.z += k * __uint_as_float(q.y << 16); a.w += k * __uint_as_float(q.y & 0xFFFF0000u);
      }
      const __nv_bfloat162 lo = __floats2bfloat162_rn(a.x, a.y), hi = __floats2bfloat162_rn(a.z, a.w);
      uint2 o;
      o.x = *reinterpret_cast<const uint32_t*>(&lo); o.y = *reinterpret_cast<const uint32_t*>(&hi);
      *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(C) + row * ldc + col) = o;
    } else {
      float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(C) + row * ldc + col);
      if (accumulate) { const float4 w = *q; a.x += w.x; a.y += w.y; a.z += w.z; a.w += w.w; }
      *q = a;
    }
  }
}

// g (EPI_CHAIN, C its final destination) in one launch, or in splits through `parts` and a summing kernel.
static int chain_gemm(GemmArgs g, float* parts, cudaStream_t s) {
  const int splits = gemm_chain_splits(g);
  if (splits == 1) return gemm_tcgen05(g, s);
  GemmArgs q = g;
  q.C = parts; q.ldc = g.N; q.c_dtype = DT_F32;
  q.epi.splits = splits; q.epi.accumulate = 0; q.epi.part_stride = (long long)g.M * g.N;
  q.epi.vh.corr = nullptr;                     // the summing kernel adds it
  const int rc = gemm_tcgen05(q, s);
  if (rc != PCM_OK) return rc;
  const long long total = (long long)g.M * (g.N / 4);
  const int grid = (int)(ceil_div(total, 256) < 8 * sm_count() ? ceil_div(total, 256) : 8 * sm_count());
  return launch_after(g.c_dtype == DT_BF16 ? parts_sum_kernel<true> : parts_sum_kernel<false>, dim3(grid), dim3(256), s, parts,
                      q.epi.part_stride, splits, g.M, g.N, g.C, g.ldc, g.epi.accumulate, g.epi.vh);
}

// Profile class of a product: on CTA pairs or not (the choice that gemm_tcgen05 makes).
static int gemm_class(long long M, long long N) { return M > 128 && N > 128 ? PC_GEMM : PC_GEMM_SMALL; }

static size_t round256(size_t v) { return (v + 255) / 256 * 256; }

struct HeadBwdPlan { size_t x, hi, lo, parts, coef, corr, sort, total; long long ldz; int rows; };
static HeadBwdPlan head_bwd_plan(int M, int d, int V, int chunk_rows) {
  HeadBwdPlan pl;
  pl.rows = chunk_rows < M ? chunk_rows : M;
  pl.ldz = ((long long)V + 31) / 32 * 32;     // whole 32-column slices of the epilogue
  pl.x = 0;
  pl.hi = round256((size_t)pl.rows * d * 2);
  pl.lo = pl.hi + round256((size_t)pl.rows * pl.ldz * 2);
  pl.parts = pl.lo + round256((size_t)pl.rows * pl.ldz * 2);
  pl.coef = pl.parts + round256(chain_part_bytes());
  pl.corr = pl.coef + round256((size_t)pl.rows * sizeof(float));
  pl.sort = pl.corr + round256((size_t)pl.rows * sizeof(float));
  pl.total = pl.sort + (pl.rows > 0 ? embed_accumulate_bytes(pl.rows, V, d) : 0);
  return pl;
}

static bool head_args_ok(const void* x, int64_t ld_x, const void* w, int64_t ld_w, int32_t d, const int32_t* tok) {
  return x && w && tok && !(((uintptr_t)x | (uintptr_t)w) & 15) && ld_x >= d && ld_w >= d;
}
// Tiles are counted in 32 bits, at 64 columns and 128 rows the smallest; so are the contraction's k-blocks, rounded up.
static bool head_shape_ok(int64_t ld_x, int64_t ld_w, int32_t d, int64_t n_rows, int64_t vocab) {
  return d % 8 == 0 && ld_x % 8 == 0 && ld_w % 8 == 0 && n_rows <= PCM_MAX_VOCAB_CALL && vocab <= PCM_MAX_VOCAB_CALL && d <= PCM_MAX_VOCAB_CALL &&
         (n_rows / 128 + 1) * (vocab / 64 + 1) < (1ll << 31) && ((int64_t)d / 64 + 1) * (vocab / 64 + 1) < (1ll << 31);
}

}  // namespace pcm

using namespace pcm;

extern "C" size_t grpo_head_logp_workspace_bytes(int32_t n_rows, int32_t d, int32_t vocab) {
  if (n_rows < 0 || d < 8 || vocab < 1 || !head_shape_ok(d, d, d, n_rows, vocab)) return 0;
  auto parts = [&](int rows) { return 2 * (size_t)ceil_div(vocab, gemm_vocab_tile(rows, vocab)) * (size_t)rows * sizeof(float4); };
  // up to 128 rows the tiles are narrower, so 128 rows can leave more parts than 129
  return round256(max(parts(n_rows), parts(min(n_rows, 128)))) + 256;
}

extern "C" int grpo_head_logp(const void* x, int64_t ld_x, int32_t n_rows, int32_t d, const void* w_h, int64_t ld_w, int32_t vocab,
                              const int32_t* tok, float temperature, float* logp, float* entropy, float* lse,
                              uint32_t* device_status, void* workspace, size_t workspace_bytes, pcm_stream stream) {
  if (n_rows < 0 || d < 1 || vocab < 1 || !vocab_temperature_ok(temperature)) return PCM_ERR_ARG;
  if (!head_shape_ok(ld_x, ld_w, d, n_rows, vocab)) return PCM_ERR_SHAPE;
  if (n_rows == 0) return PCM_OK;
  if (!head_args_ok(x, ld_x, w_h, ld_w, d, tok)) return PCM_ERR_ARG;
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < grpo_head_logp_workspace_bytes(n_rows, d, vocab)) return PCM_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  const float inv_t = 1.f / temperature;
  float4* part = (float4*)workspace;
  GemmArgs g{n_rows, vocab, d, x, ld_x, true, w_h, ld_w, true, DT_BF16, nullptr, 0, DT_BF16, nullptr, 0};
  g.epi.kind = EPI_VOCAB_STATS;
  g.epi.status = device_status;
  g.epi.vh.tok = tok; g.epi.vh.inv_t = inv_t; g.epi.vh.part = part; g.epi.vh.vocab = vocab;
  prof_begin(gemm_class(n_rows, 256), s);
  int rc = gemm_tcgen05(g, s);
  prof_end(s, 2.0 * n_rows * vocab * d, 2.0 * d * ((double)n_rows + vocab));
  if (rc != PCM_OK) return rc;
  prof_begin(PC_LOSS, s);
  const int bn = gemm_vocab_tile(n_rows, vocab);
  const JoinParams jp{part, n_rows, vocab, bn, 2 * ceil_div(vocab, bn), tok, inv_t, logp, entropy, lse, device_status};
  rc = n_rows <= 1024 ? launch_after(vocab_stats_join_row_kernel, dim3(n_rows), dim3(128), s, jp)
                      : launch_after(vocab_stats_join_kernel, dim3(ceil_div(n_rows, 32)), dim3(32 * VH_GROUPS), s, jp);
  prof_end(s, 0.0, 16.0 * n_rows * jp.parts);
  return rc;
}

extern "C" size_t grpo_head_logp_bwd_workspace_bytes(int32_t n_rows, int32_t d, int32_t vocab, int32_t chunk_rows) {
  if (n_rows < 0 || d < 8 || vocab < 1 || chunk_rows < 1 || !head_shape_ok(d, d, d, n_rows, vocab)) return 0;
  return head_bwd_plan(n_rows, d, vocab, chunk_rows).total + 256;
}

extern "C" int grpo_head_logp_bwd(const void* x, int64_t ld_x, int32_t n_rows, int32_t d, const void* w_h, int64_t ld_w,
                                  int32_t vocab, const int32_t* tok, float temperature, const float* lse, const float* entropy,
                                  const float* dlogp, const float* dentropy, int32_t chunk_rows, uint32_t flags, void* dx,
                                  int64_t ld_dx, float* dw, uint32_t* device_status, void* workspace, size_t workspace_bytes,
                                  pcm_stream stream) {
  if (n_rows < 0 || d < 1 || vocab < 1 || chunk_rows < 1 || !vocab_temperature_ok(temperature) || (flags & ~(GRPO_ACCUMULATE | GRPO_EXACT_DX))) return PCM_ERR_ARG;
  if (!head_shape_ok(ld_x, ld_w, d, n_rows, vocab) || (dx && ld_dx % 8)) return PCM_ERR_SHAPE;
  if ((!dx && !dw) || (dx && (((uintptr_t)dx & 15) || ld_dx < d)) || (dw && ((uintptr_t)dw & 15))) return PCM_ERR_ARG;
  const bool accumulate = flags & GRPO_ACCUMULATE, exact_dx = dx && (flags & GRPO_EXACT_DX);
  cudaStream_t s = (cudaStream_t)stream;
  if (n_rows == 0) {
    if (dw && !accumulate) PCM_CUDA_TRY(cudaMemsetAsync(dw, 0, (size_t)vocab * d * sizeof(float), s));
    return PCM_OK;
  }
  if (!head_args_ok(x, ld_x, w_h, ld_w, d, tok) || !lse || !dlogp || (dentropy && !entropy)) return PCM_ERR_ARG;
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < grpo_head_logp_bwd_workspace_bytes(n_rows, d, vocab, chunk_rows))
    return PCM_ERR_WORKSPACE;
  const HeadBwdPlan pl = head_bwd_plan(n_rows, d, vocab, chunk_rows);
  unsigned char* base = (unsigned char*)workspace;
  uint4* x_live = (uint4*)(base + pl.x);
  void *hi = base + pl.hi, *lo = base + pl.lo;
  float *parts = (float*)(base + pl.parts), *coef = (float*)(base + pl.coef), *corr = (float*)(base + pl.corr);
  const float inv_t = 1.f / temperature;
  for (int r0 = 0; r0 < n_rows; r0 += pl.rows) {
    const int rows = n_rows - r0 < pl.rows ? n_rows - r0 : pl.rows;
    const unsigned short* xr = (const unsigned short*)x + (long long)r0 * ld_x;
    const double flops = 2.0 * rows * vocab * d;
    int rc = PCM_OK;
    if (dw) {
      prof_begin(PC_EMBED, s);
      rc = embed_accumulate_sort(tok + r0, rows, vocab, d, base + pl.sort, pl.total - pl.sort, s);
      prof_end(s, 0.0, 4.0 * rows);
      if (rc != PCM_OK) return rc;
    }
    prof_begin(PC_ELEM, s);
    const int d8 = d / 8;
    const int blocks = ceil_div((long long)rows * d8, 1024);
    rc = launch_after(live_rows_kernel, dim3(blocks), dim3(256), s, (const uint4*)xr, ld_x / 8, rows, d8, tok + r0, lse + r0, vocab,
                      x_live, device_status, dw ? 1 : 0);
    prof_end(s, 0.0, 4.0 * rows * d);
    if (rc != PCM_OK) return rc;

    GemmArgs z{rows, vocab, d, x_live, d, true, w_h, ld_w, true, DT_BF16, hi, pl.ldz, DT_BF16, nullptr, 0};
    z.epi.kind = EPI_VOCAB_DZ;
    z.epi.status = device_status;
    VocabHeadArgs& v = z.epi.vh;
    v.tok = tok + r0; v.inv_t = inv_t; v.lse = lse + r0; v.dlogp = dlogp + r0; v.vocab = vocab; v.dz_lo = lo;
    v.coef = dw || exact_dx ? coef : nullptr;
    v.corr = dx && !exact_dx ? corr : nullptr;
    v.dent = dentropy ? dentropy + r0 : nullptr;
    v.entropy = dentropy ? entropy + r0 : nullptr;
    prof_begin(gemm_class(rows, 256), s);
    rc = gemm_tcgen05(z, s);
    prof_end(s, flops, 2.0 * d * ((double)rows + vocab) + 4.0 * rows * vocab);
    if (rc != PCM_OK) return rc;
    if (dx) {
      GemmArgs q{rows, d, vocab, hi, pl.ldz, true, w_h, ld_w, false, DT_BF16, (unsigned short*)dx + (long long)r0 * ld_dx, ld_dx, DT_BF16, nullptr, 0};
      q.epi.kind = EPI_CHAIN;                  // bf16 result: one accumulator piece
      q.epi.status = device_status;
      q.epi.vh.tok = tok + r0; q.epi.vh.vocab = vocab; q.epi.vh.corr = corr;
      if (exact_dx) {                          // hi + lo, which cancel at the targets: all of their d z is added in fp32
        q.A2 = lo; q.lda2 = pl.ldz; q.B2 = w_h; q.ldb2 = ld_w; q.K2 = vocab;
        q.epi.vh.corr = coef;
      }
      q.epi.vh.w = (const __nv_bfloat16*)w_h; q.epi.vh.ld_w = ld_w;
      prof_begin(gemm_class(rows, d), s);
      rc = chain_gemm(q, parts, s);
      prof_end(s, exact_dx ? 2.0 * flops : flops, (exact_dx ? 4.0 : 2.0) * rows * vocab + 2.0 * vocab * d + 2.0 * rows * d);
      if (rc != PCM_OK) return rc;
    }
    if (dw) {
      GemmArgs q{vocab, d, rows, hi, pl.ldz, false, x_live, d, false, DT_BF16, dw, d, DT_F32, nullptr, 0};
      q.A2 = lo; q.lda2 = pl.ldz; q.B2 = x_live; q.ldb2 = d; q.K2 = rows;
      q.epi.kind = EPI_CHAIN;
      q.epi.status = device_status;
      q.epi.chain_kb = VH_CHAIN_KB;
      q.epi.accumulate = accumulate || r0 > 0;
      prof_begin(gemm_class(vocab, d), s);
      rc = chain_gemm(q, parts, s);
      prof_end(s, 2.0 * flops, 4.0 * rows * vocab + 4.0 * rows * d + 4.0 * vocab * d);
      if (rc != PCM_OK) return rc;
      prof_begin(PC_EMBED, s);
      rc = embed_accumulate_sum(x_live, coef, rows, vocab, d, dw, base + pl.sort, s);
      prof_end(s, 2.0 * rows * d, 2.0 * rows * d);
      if (rc != PCM_OK) return rc;
    }
  }
  return PCM_OK;
}
