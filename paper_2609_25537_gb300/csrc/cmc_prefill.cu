// Norm and rotary embedding of the heads of many tokens, alone (cmc_qk_norm_rope) and with the
// append of their keys and values to the Tier-2 ring (cmc_window_prefill).
#include "cmc_prep.cuh"

namespace cmc {

constexpr int kPrefillWarps = 8;
constexpr int kPrefillBatch = 4;  // rows a lane group has in flight

struct PrefillParams {
  const uint16_t* q;  // token rows of Hq heads, q_stride elements apart; NULL: no queries
  const uint16_t* k;
  const uint16_t* v;  // NULL without a ring
  long long q_stride, k_stride, v_stride;
  uint16_t* out_q;    // [B, L, T, Hq, d]
  uint16_t* out_k;    // [B, L, T, Hkv, d] (no ring)
  uint16_t* ring_k;   // [B, L, Hkv, W, d]
  uint16_t* ring_v;
  float* ring_weight;  // [B, L, Hkv, W] or NULL
  int64_t* pos;
  const int64_t* count;  // [B] or NULL
  uint32_t* status;
  unsigned long long* tickets;
  int L, T, Hq, Hkv, W;
  int parts;  // warps that share a token's rows
  PrepParams prep;
};

// A warp takes a token's heads, or one of `parts` equal shares of them, d / 16 lanes to a head's row.
template <int D, bool RING>
__global__ void __launch_bounds__(32 * kPrefillWarps)
prefill_kernel(const __grid_constant__ PrefillParams p) {
  using P = Prep<D>;
  __shared__ float2 table[kPrefillWarps][D / 2];
  __shared__ long long pos_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int b = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x == 0) pos_s = *static_cast<volatile const int64_t*>(p.pos + b);
  __syncthreads();
  const long long pos = pos_s;
  int n = p.T;
  if (RING && p.count) {
    const long long c = p.count[b];
    n = c < 0 ? 0 : c < p.T ? static_cast<int>(c) : p.T;
  }
  if (RING && threadIdx.x == 0) {
    // the last of the sequence's CTAs to have read pos advances it
    __threadfence();
    if (atomicAdd(p.tickets + b, 1ull) + 1 == gridDim.x) {
      if (pos >= 0) p.pos[b] = pos + n;
      else atomicOr(p.status, CMC_DEVFLAG_BAD_POS);
      p.tickets[b] = 0ull;
    }
  }
  if (RING && pos < 0) return;
  const long long item = static_cast<long long>(blockIdx.x) * kPrefillWarps + warp;
  const long long tok = item / p.parts;  // l T + t
  const int part = static_cast<int>(item - tok * p.parts);
  const int l = static_cast<int>(tok / p.T);
  const int t = static_cast<int>(tok - static_cast<long long>(l) * p.T);
  if (l >= p.L || t >= n) return;
  const int c = lane % P::kLanes, sub = lane / P::kLanes;

  float2 cs[8];
  if (p.prep.rope) {
    unsigned long long at = static_cast<unsigned long long>(p.prep.rope_offset + pos + t);
    if (p.prep.evicted) at += static_cast<unsigned long long>(p.prep.evicted[b]);
    prep_table<D>(p.prep, at, lane, table[warp]);
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = table[warp][8 * c + e];
  }

  // Rows: Hq of q, Hkv of k, and with a ring Hkv of v.  Those of k and v that the ring does not
  // keep are left out.
  const bool kept = !RING || t >= n - p.W;
  long long slot = 0;
  if (RING && kept) {
    const unsigned long long at = static_cast<unsigned long long>(pos) + static_cast<unsigned long long>(t);
    slot = (at >> 32) == 0 ? static_cast<unsigned>(at) % static_cast<unsigned>(p.W)
                           : static_cast<long long>(at % static_cast<unsigned>(p.W));
  }
  const int nq = p.q ? p.Hq : 0;
  const int rows = nq + (kept ? (RING ? 2 : 1) * p.Hkv : 0);
  const int steps = (rows + P::kRows - 1) / P::kRows;
  const int per = (steps + p.parts - 1) / p.parts;
  const int s1 = min(steps, (part + 1) * per);
  const long long row0 = (static_cast<long long>(b) * p.L + l) * p.T + t;
  const uint16_t* qrow = p.q + row0 * p.q_stride;
  const uint16_t* krow = p.k + row0 * p.k_stride;
  const uint16_t* vrow = RING ? p.v + row0 * p.v_stride : nullptr;
  const long long unit0 = (static_cast<long long>(b) * p.L + l) * p.Hkv;
  for (int s0 = part * per; s0 < s1; s0 += kPrefillBatch) {
    uint4 a[kPrefillBatch][2];
#pragma unroll
    for (int e = 0; e < kPrefillBatch; ++e) {
      const int r = (s0 + e) * P::kRows + sub;
      a[e][0] = a[e][1] = make_uint4(0u, 0u, 0u, 0u);
      if (s0 + e < s1 && r < rows) {
        const uint16_t* src = r < nq             ? qrow + static_cast<long long>(r) * D
                              : r < nq + p.Hkv ? krow + static_cast<long long>(r - nq) * D
                                               : vrow + static_cast<long long>(r - nq - p.Hkv) * D;
        a[e][0] = *reinterpret_cast<const uint4*>(src + 8 * c);
        a[e][1] = *reinterpret_cast<const uint4*>(src + D / 2 + 8 * c);
      }
    }
#pragma unroll
    for (int e = 0; e < kPrefillBatch; ++e) {
      if (s0 + e >= s1) break;
      const int r = (s0 + e) * P::kRows + sub;
      const int h = r < nq ? r : r < nq + p.Hkv ? r - nq : r - nq - p.Hkv;
      const bool is_v = r >= nq + p.Hkv;
      float x[16];
      prep_unpack(a[e][0], a[e][1], x);
      const float* w = is_v ? nullptr : r < nq ? p.prep.q_weight : p.prep.k_weight;
      float4 gain[4];
      if (w) prep_gains<D>(w + static_cast<long long>(l) * D, c, gain);
      prep_norm<D>(x, gain, w != nullptr, p.prep.eps);
      if (p.prep.rope) prep_rotate(x, cs);
      if (!is_v) {
        a[e][0] = prep_pack(x);
        a[e][1] = prep_pack(x + 8);
      }
      if (r < rows) {
        uint16_t* dst;
        if (r < nq) dst = p.out_q + (row0 * p.Hq + h) * D;
        else if (RING) dst = (is_v ? p.ring_v : p.ring_k) + ((unit0 + h) * p.W + slot) * D;
        else dst = p.out_k + (row0 * p.Hkv + h) * D;
        *reinterpret_cast<uint4*>(dst + 8 * c) = a[e][0];
        *reinterpret_cast<uint4*>(dst + D / 2 + 8 * c) = a[e][1];
        if (RING && is_v && c == 0 && p.ring_weight) p.ring_weight[(unit0 + h) * p.W + slot] = 0.f;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

static int run_prefill(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                       int64_t v_stride, int T, void* ring_k, void* ring_v, float* ring_weight,
                       int64_t* pos, const int64_t* count, const cmc_dims* dims, const cmc_qk_prep* prep,
                       void* out_q, void* out_k, void* workspace, size_t workspace_bytes, bool ring,
                       void* stream) {
  if (!dims) return CMC_ERR_NULL;
  cmc_dims m = *dims;
  if (!ring) m.W = 1;
  m.N = 1;
  m.k = 0;
  int st = validate_dims(&m, true);
  if (st != CMC_OK) return st;
  if (T < 0 || T > (1 << 24)) return CMC_ERR_SHAPE;
  if (T == 0) return CMC_OK;  // pointers of empty tensors may be NULL
  const long long items = static_cast<long long>(m.L) * T;
  if (items >= (1LL << 27)) return CMC_ERR_SHAPE;
  if (!k || !pos || (!ring && (!q || !out_q || !out_k)) || (q && !out_q)) return CMC_ERR_NULL;
  if (ring && (!v || !ring_k || !ring_v)) return CMC_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out_q) || !aligned16(out_k) ||
      !aligned16(ring_k) || !aligned16(ring_v) || (reinterpret_cast<uintptr_t>(ring_weight) & 3) ||
      ((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(count)) & 7))
    return CMC_ERR_ALIGN;
  const long long qd = static_cast<long long>(m.Hq) * m.d, kd = static_cast<long long>(m.Hkv) * m.d;
  if ((q && q_stride < qd) || k_stride < kd || (ring && v_stride < kd)) return CMC_ERR_SHAPE;
  if (((q ? q_stride : 0) | k_stride | (ring ? v_stride : 0)) & 7) return CMC_ERR_ALIGN;
  if (ring) {
    if (!workspace || workspace_bytes < ws_partials_off(m.B)) return CMC_ERR_WORKSPACE;
    if (!aligned16(workspace)) return CMC_ERR_ALIGN;
  }
  PrefillParams p;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  st = prep_params(prep, m.d, s, &p.prep);
  if (st != CMC_OK) return st;
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.out_q = static_cast<uint16_t*>(out_q);
  p.out_k = static_cast<uint16_t*>(out_k);
  p.ring_k = static_cast<uint16_t*>(ring_k);
  p.ring_v = static_cast<uint16_t*>(ring_v);
  p.ring_weight = ring_weight;
  p.pos = pos;
  p.count = count;
  char* ws = static_cast<char*>(workspace);
  p.status = reinterpret_cast<uint32_t*>(ws);
  p.tickets = ring ? reinterpret_cast<unsigned long long*>(ws + kWsHeader) : nullptr;
  p.L = m.L; p.T = T; p.Hq = m.Hq; p.Hkv = m.Hkv; p.W = m.W;
  // Few tokens: a token's rows are shared out over more warps, down to one step each.
  const int rows_at_once = m.d == 128 ? Prep<128>::kRows : Prep<64>::kRows;
  const int steps = ((q ? m.Hq : 0) + (ring ? 2 : 1) * m.Hkv + rows_at_once - 1) / rows_at_once;
  const long long wanted = 16LL * sm_count() / (items * m.B);
  p.parts = static_cast<int>(wanted < 1 ? 1 : wanted > steps ? steps : wanted);
  const long long ctas = (items * p.parts + kPrefillWarps - 1) / kPrefillWarps;
  const dim3 grid(static_cast<unsigned>(ctas), static_cast<unsigned>(m.B));
  auto kern = ring ? (m.d == 128 ? prefill_kernel<128, true> : prefill_kernel<64, true>)
                   : (m.d == 128 ? prefill_kernel<128, false> : prefill_kernel<64, false>);
  return launch_pdl(kern, grid, dim3(32 * kPrefillWarps), 0, s, p);
}

}  // namespace cmc

extern "C" {

size_t cmc_cache_workspace_size(int B) { return B < 1 || B > 65535 ? 0 : cmc::ws_partials_off(B); }

int cmc_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, int T,
                     const int64_t* pos, const cmc_dims* dims, const cmc_qk_prep* prep, void* out_q,
                     void* out_k, void* stream) {
  return cmc::run_prefill(q, q_stride, k, k_stride, nullptr, 0, T, nullptr, nullptr, nullptr,
                          const_cast<int64_t*>(pos), nullptr, dims, prep, out_q, out_k, nullptr, 0, false,
                          stream);
}

int cmc_window_prefill(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                       int64_t v_stride, int T, void* ring_k, void* ring_v, float* ring_weight,
                       int64_t* pos, const int64_t* count, const cmc_dims* dims, const cmc_qk_prep* prep,
                       void* out_q, void* workspace, size_t workspace_bytes, void* stream) {
  return cmc::run_prefill(q, q_stride, k, k_stride, v, v_stride, T, ring_k, ring_v, ring_weight, pos,
                          count, dims, prep, out_q, nullptr, workspace, workspace_bytes, true, stream);
}

}  // extern "C"
