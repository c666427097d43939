// Norm and rotary embedding of query and key heads, shared by cmc_qk_norm_rope and
// cmc_window_prefill (cmc_prefill.cu) and by the fused step of cmc_attn_weighted.cu:
//   y = x / sqrt(mean(x^2) + eps) * w          (RMS norm of one head, where w is given)
//   out_i       = y_i cos a_i - y_(i + d/2) sin a_i
//   out_(i+d/2) = y_(i + d/2) cos a_i + y_i sin a_i,   a_i = p theta^(-2i/d)
// all in fp32; the caller rounds once, to bf16 (a model that rounds between the two has one
// rounding more).
//
// A head's row is taken by d / 16 lanes: lane c of them has 16-byte chunks c and c + d / 16, which are
// elements 8 c .. 8 c + 7 and their partners d / 2 further on, so that the rotation needs nothing from
// another lane and the norm one sum over the group.
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

template <int D>
struct Prep {
  static constexpr int kLanes = D / 16;         // lanes of one row
  static constexpr int kRows = 32 / kLanes;     // rows that a warp takes at once
};

// (cos, sin) of the d / 2 pairs at position p, into the warp's table.  The caller's __syncwarp
// lets the warp read it.
template <int D>
__device__ __forceinline__ void prep_table(const PrepParams& p, unsigned long long at, int lane, float2* tab) {
#pragma unroll
  for (int e = 0; e < D / 64; ++e) {
    const int i = lane + 32 * e;
    const unsigned long long turns =
        p.rope_slot >= 0 ? g_rope_tables[p.rope_slot][i] : p.rope_turns[i];
    tab[i] = rope_cos_sin(at, turns);
  }
}

// A lane's share of a row of gains.
template <int D>
__device__ __forceinline__ void prep_gains(const float* w, int c, float4 (&g)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) g[e] = *reinterpret_cast<const float4*>(w + (e >> 1) * (D / 2) + 8 * c + 4 * (e & 1));
}

// One row's share of a lane: x[0..7] and x[8..15] are elements 8 c .. and d / 2 + 8 c ...  `norm` differs
// between the rows of a warp, all of whose lanes take part.
template <int D>
__device__ __forceinline__ void prep_norm(float (&x)[16], const float4 (&g)[4], bool norm, float eps) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) s = fmaf(x[e], x[e], s);
#pragma unroll
  for (int off = 1; off < Prep<D>::kLanes; off <<= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  if (!norm) return;
  const float r = 1.f / sqrtf(fmaf(s, 1.f / D, eps));
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[4 * e + 0] *= r * g[e].x;
    x[4 * e + 1] *= r * g[e].y;
    x[4 * e + 2] *= r * g[e].z;
    x[4 * e + 3] *= r * g[e].w;
  }
}

// cs: (cos, sin) of pairs 8 c .. 8 c + 7.
__device__ __forceinline__ void prep_rotate(float (&x)[16], const float2 (&cs)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float lo = x[e], hi = x[8 + e];
    x[e] = fmaf(lo, cs[e].x, -hi * cs[e].y);
    x[8 + e] = fmaf(hi, cs[e].x, lo * cs[e].y);
  }
}

__device__ __forceinline__ void prep_unpack(const uint4& lo, const uint4& hi, float (&x)[16]) {
  float a[8], b[8];
  unpack8(lo, a);
  unpack8(hi, b);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = a[e];
    x[8 + e] = b[e];
  }
}

__device__ __forceinline__ uint4 prep_pack(const float* x) {
  return make_uint4(pack_bf16_rn(x[0], x[1]), pack_bf16_rn(x[2], x[3]), pack_bf16_rn(x[4], x[5]),
                    pack_bf16_rn(x[6], x[7]));
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// Checks a cmc_qk_prep (NULL: neither norm nor rotation) and fills in the launch's parameters.
static int prep_params(const cmc_qk_prep* q, int d, cudaStream_t s, PrepParams* p) {
  memset(p, 0, sizeof(*p));
  p->rope_slot = -1;
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
    rope_turns_table(q->rope_theta, d, p->rope_turns);
    p->rope_slot = rope_slot(q->rope_theta, d, p->rope_turns, s);
  }
  return CMC_OK;
}

}  // namespace cmc
