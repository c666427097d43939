// Norm and rotary embedding of query and key heads, shared by cmc_qk_norm_rope and
// cmc_window_prefill (cmc_prefill.cu) and by the fused step of cmc_attn_weighted.cu:
//   y = x / sqrt(mean(x^2) + eps) * w          (RMS norm of one head, where w is given)
//   out_i       = y_i cos a_i - y_(i + d/2) sin a_i
//   out_(i+d/2) = y_(i + d/2) cos a_i + y_i sin a_i,   a_i = p theta^(-2i/d)
// all in fp32; the caller rounds once, to bf16 (a model that rounds between the two has one
// rounding more).  The callers have a row in different lanes, d / 16 or d / 4 to a row, and take the same steps.
#pragma once

#include "cmc_attn.cuh"

namespace cmc {

// Per call: what cmc_qk_prep says, checked.
struct PrepParams {
  const float* q_weight;  // [L, d] or NULL
  const float* k_weight;
  const int64_t* evicted;  // [B] or NULL
  float eps;
  int rope;               // 0: no rotation
  int rope_slot;          // >= 0: the table in g_rope_tables, else rope_turns
  long long rope_offset;
  unsigned long long rope_turns[64];
};

// ---------------------------------------------------------------------------
// Device side: the arithmetic, operation by operation, so that a token has the same key bit for bit whichever call prepares it
// ---------------------------------------------------------------------------

// Sum of squares of a row.  Quad j, elements 2 j, 2 j + 1 and their partners d / 2 further on, in this order; the d / 4 quads in a
// tree of neighbours: 0 with 1, 2 with 3, then their sums, and so on (a butterfly over lanes gives all of them the same).
__device__ __forceinline__ float quad_squares(float x0, float x1, float y0, float y1) {
  return fmaf(y1, y1, fmaf(y0, y0, fmaf(x1, x1, __fmul_rn(x0, x0))));
}

// Mean of squares + eps, of a row whose elements were taken `by` times as large; 1 / sqrt of it is the row's factor (rsqrtf: 2^-22).
template <int D>
__device__ __forceinline__ float row_mean(float squares, float eps, float by = 1.f) {
  return fmaf(squares, 1.f / D, __fmul_rn(__fmul_rn(eps, by), by));
}

// Squares of elements of 2^60 and more may add up to infinity, and those of a row below 2^-45 lose their bits where no eps counts
// more.  A mean that is then infinite, below 2^-96 or NaN shows it: the squares are summed once more of elements taken 2^-70 or 2^80
// times as large (what 2^-70 leaves nothing of counts nothing in such a sum), and the smallest rows stay 2^80 times as large, since
// their factor may be more than fp32 holds.
constexpr uint32_t kOddMean = 0x0F800000u, kOddMeans = 0x7F800000u - kOddMean;  // 2^-96, and how many floats there are from it to infinity
__device__ __forceinline__ bool odd_mean(float mean) { return __float_as_uint(mean) - kOddMean >= kOddMeans; }
__device__ __forceinline__ float odd_scale(float mean) { return mean < 1.f ? 0x1p80f : 0x1p-70f; }

// What a pair's gains g, h and its angle make of it: (g cos a, h sin a, h cos a, g sin a).
__device__ __forceinline__ float4 pair_factors(float g, float h, float2 cos_sin) {
  return make_float4(__fmul_rn(g, cos_sin.x), __fmul_rn(h, cos_sin.y), __fmul_rn(h, cos_sin.x), __fmul_rn(g, cos_sin.y));
}

// Elements x and y of a pair, by their row's factor r and the pair's t.
__device__ __forceinline__ void prep_pair(float& x, float& y, float r, bool rope, const float4& t) {
  const float u = __fmul_rn(r, x), v = __fmul_rn(r, y);
  x = rope ? fmaf(u, t.x, -__fmul_rn(v, t.y)) : __fmul_rn(u, t.x);
  y = rope ? fmaf(v, t.z, __fmul_rn(u, t.w)) : __fmul_rn(v, t.z);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// The device table of (theta, d), as rope_slot finds it; the last one that a thread asked for is found without its locks
// (a slot once written stays as it is).
static int rope_slot_again(double theta, int d, cudaStream_t s, unsigned long long (&turns)[64]) {
  struct Last {
    double theta;
    int d, dev, slot;
  };
  static thread_local Last last = {0.0, 0, -1, -1};
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    dev = -1;
  }
  if (dev >= 0 && last.dev == dev && last.d == d && last.theta == theta) return last.slot;
  rope_turns_table(theta, d, turns);
  const int slot = rope_slot(theta, d, turns, s);
  if (slot >= 0) last = {theta, d, dev, slot};
  return slot;
}

// Checks a cmc_qk_prep (NULL: neither norm nor rotation) and fills in the launch's parameters (rope_turns only where there is
// no device table).
static int prep_params(const cmc_qk_prep* q, int d, cudaStream_t s, PrepParams* p) {
  p->q_weight = p->k_weight = nullptr;
  p->evicted = nullptr;
  p->eps = 0.f;
  p->rope = 0;
  p->rope_slot = -1;
  p->rope_offset = 0;
  if (!q) return CMC_OK;
  if (!aligned16(q->q_weight) || !aligned16(q->k_weight) ||
      (reinterpret_cast<uintptr_t>(q->evicted) & 7))
    return CMC_ERR_ALIGN;
  if ((q->q_weight || q->k_weight) && !(q->eps >= 0.f && q->eps < INFINITY)) return CMC_ERR_RANGE;
  p->q_weight = q->q_weight;
  p->k_weight = q->k_weight;
  p->eps = q->eps;
  p->evicted = q->evicted;
  if (q->rope_theta != 0.0) {
    if (!(q->rope_theta > 0.0 && q->rope_theta < 1e300)) return CMC_ERR_RANGE;
    if (q->rope_offset < 0 || q->rope_offset > (1LL << 32)) return CMC_ERR_RANGE;
    p->rope = 1;
    p->rope_offset = q->rope_offset;
    p->rope_slot = rope_slot_again(q->rope_theta, d, s, p->rope_turns);
  }
  return CMC_OK;
}

}  // namespace cmc
