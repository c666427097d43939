// Decode attention over the two-tier cache held in 8 bits (format: cmc_q8.cuh).
//
// One CTA per unit (sequence, layer, KV head); its four warps take every fourth
// key of [Tier-1 | live ring slots] each and keep an online softmax of the G
// query heads in fp32; the warps' states are merged in shared memory.
#include "cmc_attn.cuh"
#include "cmc_q8.cuh"

namespace cmc {

struct Q8Params {
  const uint16_t* q;
  const uint8_t *t1_kv, *t1_scales, *ring_kv, *ring_scales;
  const int64_t* pos;
  uint16_t* out;
  uint32_t* status;
  int G, LH, N, k, W, t1S, ringS;
  float scale_log2;
};

template <int D, int G>
__global__ void __launch_bounds__(kThreads)
attn_q8_kernel(const Q8Params p) {
  constexpr int E = D / 32;
  __shared__ float sm[kWarps][8], sl[kWarps][8], so[kWarps][G][D];
  pdl_wait();
  pdl_trigger();
  const int u = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long pb = p.pos[u / p.LH];
  const int n1 = pb < 0 ? 0 : p.k, n2 = pb < 0 ? 0 : static_cast<int>(pb < p.W ? pb : p.W);
  if (pb < 0 && threadIdx.x == 0) atomicOr(p.status, CMC_DEVFLAG_BAD_POS);
  float q[G][E], o[G][E], m[G], l[G];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    m[h] = -INFINITY;
    l[h] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[h][e] = bf16lo_to_f32(p.q[(static_cast<long long>(u) * G + h) * D + lane * E + e]);
      o[h][e] = 0.f;
    }
  }
  for (int i = warp; i < n1 + n2; i += kWarps) {
    const bool t1 = i < n1;
    const int r = t1 ? i : i - n1;
    const long long T = t1 ? p.N : p.W, S = t1 ? p.t1S : p.ringS;
    const uint8_t* kv = t1 ? p.t1_kv : p.ring_kv;
    const uint8_t* sc = t1 ? p.t1_scales : p.ring_scales;
    float kx[4], vx[4];
    uint32_t kw = 0u, vw = 0u;
    for (int e = 0; e < E; ++e) {
      kw |= static_cast<uint32_t>(kv[(2LL * u * T + r) * D + lane * E + e]) << (8 * e);
      vw |= static_cast<uint32_t>(kv[((2LL * u + 1) * T + r) * D + lane * E + e]) << (8 * e);
    }
    decode4(kw, kx);
    decode4(vw, vx);
    const float ks = e8m0_to_f32(sc[2LL * u * S + r / kQ8Block]);
    const float vs = e8m0_to_f32(sc[(2LL * u + 1) * S + r / kQ8Block]);
#pragma unroll
    for (int h = 0; h < G; ++h) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s = fmaf(q[h][e], kx[e], s);
      for (int off = 1; off < 32; off <<= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
      s *= ks * p.scale_log2;
      const float mn = fmaxf(m[h], s);
      const float mr = mn == -INFINITY ? 0.f : mn;
      const float a = exp2f(m[h] - mr), w = exp2f(s - mr);
      m[h] = mn;
      l[h] = l[h] * a + w;
#pragma unroll
      for (int e = 0; e < E; ++e) o[h][e] = fmaf(w, vx[e] * vs, o[h][e] * a);
    }
  }
#pragma unroll
  for (int h = 0; h < G; ++h) {
    if (lane == 0) {
      sm[warp][h] = m[h];
      sl[warp][h] = l[h];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) so[warp][h][lane * E + e] = o[h][e];
  }
  __syncthreads();
  for (int x = threadIdx.x; x < G * D; x += kThreads) {
    const int h = x / D, c = x % D;
    float M = -INFINITY, L = 0.f, O = 0.f;
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm[w][h]);
    if (M == -INFINITY) M = 0.f;
    for (int w = 0; w < kWarps; ++w) {
      const float f = exp2f(sm[w][h] - M);
      L = fmaf(f, sl[w][h], L);
      O = fmaf(f, so[w][h][c], O);
    }
    p.out[static_cast<long long>(u) * G * D + x] = static_cast<uint16_t>(f32_to_bf16_bits(L > 0.f ? O / L : O * 0.f));
  }
}

static int run_attention_q8(const void* q, const void* t1_kv, const void* t1_scales, const void* ring_kv,
                            const void* ring_scales, const int64_t* pos, const cmc_dims* dims,
                            float scale, void* out, void* workspace, size_t workspace_bytes,
                            void* stream) {
  const cmc_dims& m = *dims;
  Q8Params p;
  p.q = static_cast<const uint16_t*>(q);
  p.t1_kv = static_cast<const uint8_t*>(t1_kv);
  p.t1_scales = static_cast<const uint8_t*>(t1_scales);
  p.ring_kv = static_cast<const uint8_t*>(ring_kv);
  p.ring_scales = static_cast<const uint8_t*>(ring_scales);
  p.pos = pos;
  p.out = static_cast<uint16_t*>(out);
  p.status = static_cast<uint32_t*>(workspace);
  p.G = m.Hq / m.Hkv; p.LH = m.L * m.Hkv; p.N = m.N; p.k = m.k; p.W = m.W;
  p.t1S = q8_scale_bytes(m.N);
  p.ringS = q8_scale_bytes(m.W);
  p.scale_log2 = (scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(m.d))) * 1.4426950408889634f;
  auto kern = m.d == 128 ? (p.G == 1 ? attn_q8_kernel<128, 1> : p.G == 2 ? attn_q8_kernel<128, 2>
                            : p.G == 4 ? attn_q8_kernel<128, 4> : attn_q8_kernel<128, 8>)
                         : (p.G == 1 ? attn_q8_kernel<64, 1> : p.G == 2 ? attn_q8_kernel<64, 2>
                            : p.G == 4 ? attn_q8_kernel<64, 4> : attn_q8_kernel<64, 8>);
  return launch_pdl(kern, dim3(static_cast<unsigned>(m.B * m.L * m.Hkv)), dim3(kThreads), 0,
                    static_cast<cudaStream_t>(stream), p);
}

static int check_q8(const void* q, const void* t1_kv, const void* t1_scales, const void* ring_kv,
                    const void* ring_scales, const int64_t* pos, const void* k_new, const void* v_new,
                    bool fused, const cmc_dims* dims, void* out, void* workspace, size_t bytes) {
  int st = validate_dims(dims, true);
  if (st != CMC_OK) return st;
  if (!q || !ring_kv || !ring_scales || !pos || !out) return CMC_ERR_NULL;
  if (dims->k > 0 && (!t1_kv || !t1_scales)) return CMC_ERR_NULL;
  if (fused && (!k_new || !v_new)) return CMC_ERR_NULL;
  if (!aligned16(q) || !aligned16(t1_kv) || !aligned16(t1_scales) || !aligned16(ring_kv) ||
      !aligned16(ring_scales) || !aligned16(out) || (reinterpret_cast<uintptr_t>(pos) & 7))
    return CMC_ERR_ALIGN;
  if (fused && (!aligned16(k_new) || !aligned16(v_new))) return CMC_ERR_ALIGN;
  if (!workspace || bytes < cmc_decode_attn_workspace_size(dims)) return CMC_ERR_WORKSPACE;
  return aligned16(workspace) ? CMC_OK : CMC_ERR_ALIGN;
}

}  // namespace cmc

extern "C" {

int cmc_two_tier_decode_attn_q8(const void* q, const void* tier1_kv, const void* tier1_scales,
                                const void* ring_kv, const void* ring_scales, const int64_t* pos,
                                const cmc_dims* dims, float scale, void* out, void* workspace,
                                size_t workspace_bytes, void* stream) {
  using namespace cmc;
  int st = check_q8(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, nullptr, nullptr, false, dims,
                    out, workspace, workspace_bytes);
  if (st != CMC_OK) return st;
  return run_attention_q8(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, dims, scale, out,
                          workspace, workspace_bytes, stream);
}

}  // extern "C"
