// Softmax statistics over a vocabulary that is seen in parts (threads, cluster ranks, accumulator tiles), shared by the
// kernels that read logits and by the GEMM epilogues that never store them.
#pragma once
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

namespace pcm {

constexpr float VOCAB_LOG2E = 1.44269504088896340736f;
constexpr float VOCAB_LN2 = 0.69314718055994530942f;

// The kernels scale logits by 1 / T and exponents by log2(e) / T, in fp32: an infinite factor would make 0 * inf of the largest
// logit of a row.
static inline bool vocab_temperature_ok(float t) { return t > 0.f && t < INFINITY && 1.f / t * VOCAB_LOG2E < INFINITY; }

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two fp32 lanes of one 64-bit register: half the issue slots of scalar adds and products.
__device__ __forceinline__ unsigned long long pack2(float a, float b) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(unsigned long long v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// Softmax statistics of a part of a row: m the largest logit, s = sum 2^t and w = sum 2^t t with t = (z - m) c,
// c = log2(e) / temperature.  t is held at -1000 or above, so that a masked logit (-inf, or the type's lowest
// value) adds 2^t = 0 to both sums instead of 0 * -inf.
struct VocabStat { float m, s, w; };

__device__ __forceinline__ VocabStat stat_join(const VocabStat& a, const VocabStat& b, float c) {
  const float m = max_nan(a.m, b.m);
  // equal maxima (two empty parts with -inf, or twice +inf) shift by nothing
  const float da = a.m == m ? 0.f : fmaxf((a.m - m) * c, -1000.f), db = b.m == m ? 0.f : fmaxf((b.m - m) * c, -1000.f);
  const float fa = ex2(da), fb = ex2(db);
  return VocabStat{m, a.s * fa + b.s * fb, fa * (a.w + a.s * da) + fb * (b.w + b.s * db)};
}

// Everything of one row that follows from its statistics.  A row whose logits are all -inf carries no distribution:
// lse = -inf, entropy 0.  A NaN or +inf among them makes both NaN.
struct RowResult {
  float m, log_s, inv_t, lse, entropy;
  __device__ RowResult(const VocabStat& st, float inv_t_) : m(st.m), log_s(0.f), inv_t(inv_t_), lse(st.m), entropy(0.f) {
    if (m == -INFINITY) return;
    if (!(m < INFINITY)) { m = lse = entropy = __uint_as_float(0x7FFFFFFFu); return; }
    log_s = logf(st.s);
    lse = m * inv_t + log_s;
    entropy = log_s - (st.w / st.s) * VOCAB_LN2;
  }
  // z - m first: large logits do not swallow the logarithm
  __device__ float logp(float z) const { return m == -INFINITY ? -INFINITY : (z - m) * inv_t - log_s; }
};

// d loss / d z of one logit z (unscaled): (1/T) (g (1[target] - p) - h p (log p + H)) with gt = g / T, ht = h / T.
// A masked logit has p = 0 and log p = -inf: nothing but a target's own term is left.
__device__ __forceinline__ float vocab_slope(float z, float inv_t, float lse, float entropy, float gt, float ht, bool is_target) {
  const float lp = z * inv_t - lse;
  const float pr = __expf(lp);
  const float r = pr == 0.f ? 0.f : -pr * (gt + ht * (lp + entropy));
  return is_target ? r + gt : r;
}

// What the head GEMM's epilogues over a wide vocabulary take and give, per row of the product.
struct VocabHeadArgs {
  const int* tok = nullptr;                   // [M]
  float inv_t = 1.f;
  float4* part = nullptr;                     // EPI_VOCAB_STATS out: [2 tiles][M] {m, s, w, the target's logit}
  const float* lse = nullptr;                 // EPI_VOCAB_DZ
  const float* entropy = nullptr;
  const float* dlogp = nullptr;
  const float* dent = nullptr;                // may be null
  void* dz_lo = nullptr;                      // bf16, laid out like C: what the bf16 rounding of C leaves
  float* coef = nullptr;                      // [M] out, may be null: d z of the row's token; dz_lo is minus C there
  float* corr = nullptr;                      // [M] what the bf16 rounding of C leaves of the token's d z: out of EPI_VOCAB_DZ (may
                                              // be null), into the EPI_CHAIN product with w, which adds corr w[tok] to its rows
  const __nv_bfloat16* w = nullptr; long long ld_w = 0;
  int vocab = 0;
};

}  // namespace pcm
