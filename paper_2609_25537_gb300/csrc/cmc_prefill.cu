// Norm and rotary embedding of the heads of many tokens, alone (cmc_qk_norm_rope) and with the
// append of their keys and values to the Tier-2 ring (cmc_window_prefill).
//
// Bound: HBM, every head's row read once and written once (4 d bytes against some 10 d flops).  A warp takes a
// token: what its position and the layer's gains make of a row goes to shared memory once, then its heads' rows pass through
// registers.  What limits the rate beside HBM is the instructions of a row, and rows on their way: 8 sequences of 4,096 tokens
// of 32 + 2 x 8 heads of 128 into rings of 2,048 slots, us a launch at two rows a lane group and 8 CTAs of four warps an SM 110.5 (91 %
// of the copy rate), three and 6 112, two and 6 120, one and 8 123; 8,192 tokens' queries and keys alone 31.4 (80 %).
#include "cmc_prep.cuh"
#include "cmc_ranges.cuh"

namespace cmc {

constexpr int kPrefillWarps = 4;
constexpr int kPrefillPerSm = 8;  // CTAs on an SM, by registers
constexpr int kPrefillBatch = 2;  // rows a lane group has in flight

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

// A head's row is taken by d / 16 lanes: lane c of them has 16-byte chunks c and c + d / 16, which are
// elements 8 c .. 8 c + 7 and their partners d / 2 further on, so that the rotation needs nothing from
// another lane and the norm one sum over the group.
template <int D>
struct Prep {
  static constexpr int kLanes = D / 16;         // lanes of one row
  static constexpr int kRows = 32 / kLanes;     // rows that a warp takes at once
};

// What the rows of a token have in common, in shared memory, a warp's own: for pair i, with gains g and h of its
// elements, (g cos a, h sin a, h cos a, g sin a) for the queries and for the keys.  In the order in which the lanes of a row read
// it, so that they do not meet in a bank (side by side as the elements are, that was what bound the kernel: 88 % of L1's
// rate, 42 us for 8,192 tokens of 32 + 8 heads).
template <int D>
struct __align__(16) TokenTable {
  float4 pair[2][8][Prep<D>::kLanes];  // [queries, keys][e][c]: pair 8 c + e
};

// Two chunks of a row, in place, by its factor r.
template <int D>
__device__ __forceinline__ void prep_chunks(uint4 (&a)[2], float r, bool rope, const float4 (&pair)[8][Prep<D>::kLanes], int c) {
  uint32_t* lo = reinterpret_cast<uint32_t*>(&a[0]);
  uint32_t* hi = reinterpret_cast<uint32_t*>(&a[1]);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float x[2] = {bf16lo_to_f32(lo[q]), bf16hi_to_f32(lo[q])}, y[2] = {bf16lo_to_f32(hi[q]), bf16hi_to_f32(hi[q])};
#pragma unroll
    for (int e = 0; e < 2; ++e) prep_pair(x[e], y[e], r, rope, pair[2 * q + e][c]);
    lo[q] = pack_bf16_rn(x[0], x[1]);
    hi[q] = pack_bf16_rn(y[0], y[1]);
  }
}

// The sum of squares of a row taken `by` times as large, given to all of its lanes, four quads each.
template <int D>
__device__ __forceinline__ float prep_squares(const uint4& a, const uint4& b, float by) {
  const uint32_t* lo = reinterpret_cast<const uint32_t*>(&a);
  const uint32_t* hi = reinterpret_cast<const uint32_t*>(&b);
  float quad[4];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    quad[q] = quad_squares(by * bf16lo_to_f32(lo[q]), by * bf16hi_to_f32(lo[q]), by * bf16lo_to_f32(hi[q]), by * bf16hi_to_f32(hi[q]));
  float s = (quad[0] + quad[1]) + (quad[2] + quad[3]);
#pragma unroll
  for (int off = 1; off < Prep<D>::kLanes; off <<= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  return s;
}

// The factor of a row whose mean is odd (all of a warp's lanes come here, for the sum); one of the smallest elements is taken 2^80 times
// as large.
template <int D>
__device__ __forceinline__ float prep_odd_row(uint4 (&a)[2], float mean, float eps) {
  const float by = odd_scale(mean);
  const float f = rsqrtf(row_mean<D>(prep_squares<D>(a[0], a[1], by), eps, by));
  if (by < 1.f) return f * by;
  if (odd_mean(mean)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t* x = reinterpret_cast<uint32_t*>(&a[h]);
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = pack_bf16_rn(by * bf16lo_to_f32(x[q]), by * bf16hi_to_f32(x[q]));
    }
  }
  return f;
}

// A warp takes a token's heads, or one of `parts` equal shares of them, d / 16 lanes to a head's row.  Rows whose mean is odd: an
// instruction a row keeps the oddest mean, and a warp that has met one takes its rows again in the end, which costs nothing that can be
// measured.  Where rows are written over (PLACE: queries or keys prepared where they are) each is looked at at once, with a vote, which
// also spills 8 to 28 bytes at the 64 registers that eight CTAs leave: 8 sequences of 4,096 tokens 117 us for 110.5, of 1,024 without a
// ring 33.5 for 31.5.
template <int D, bool RING, bool PLACE>
__global__ void __launch_bounds__(32 * kPrefillWarps, kPrefillPerSm)
prefill_kernel(const __grid_constant__ PrefillParams p) {
  using P = Prep<D>;
  __shared__ TokenTable<D> tables[kPrefillWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = lane % P::kLanes, sub = lane / P::kLanes;
  TokenTable<D>& table = tables[warp];
  const int b = blockIdx.y;
  const unsigned item = blockIdx.x * kPrefillWarps + warp;
  const unsigned tok = item / static_cast<unsigned>(p.parts);  // l T + t
  const int part = static_cast<int>(item - tok * p.parts);
  const int l = static_cast<int>(tok / static_cast<unsigned>(p.T));
  const int t = static_cast<int>(tok - static_cast<unsigned>(l) * p.T);
  // Rows: Hq of q, Hkv of k, and with a ring Hkv of v.
  const int nq = p.q ? p.Hq : 0;
  const int all = nq + (RING ? 2 : 1) * p.Hkv;
  const int per = ((all + P::kRows - 1) / P::kRows + p.parts - 1) / p.parts;  // steps of a warp
  const int first = part * per;
  const long long row0 = (static_cast<long long>(b) * p.L + l) * p.T + t;
  const uint16_t* qrow = p.q + row0 * p.q_stride + 8 * c;
  const uint16_t* krow = p.k + row0 * p.k_stride + 8 * c;
  const uint16_t* vrow = p.v + row0 * p.v_stride + 8 * c;
  unsigned long long turns[D / 64];
  if (p.prep.rope)
#pragma unroll
    for (int e = 0; e < D / 64; ++e)
      turns[e] = p.prep.rope_slot >= 0 ? g_rope_tables[p.prep.rope_slot][lane + 32 * e] : p.prep.rope_turns[lane + 32 * e];
  pdl_wait();
  pdl_trigger();

  // Everything that comes before the first rows' arithmetic is requested together, the first rows with it where their
  // number does not depend on what is read.
  const long long pos = *static_cast<volatile const int64_t*>(p.pos + b);
  const long long moved = p.prep.evicted ? p.prep.evicted[b] : 0;
  long long count = p.T;
  if (RING && p.count) count = p.count[b];
  uint4 a[kPrefillBatch][2];
  auto load = [&](int s0, int end, int rows) {
#pragma unroll
    for (int e = 0; e < kPrefillBatch; ++e) {
      const int r = (s0 + e) * P::kRows + sub;
      a[e][0] = a[e][1] = make_uint4(0u, 0u, 0u, 0u);
      if (s0 + e < end && r < rows) {
        const uint16_t* src = r < nq             ? qrow + r * D
                              : r < nq + p.Hkv ? krow + (r - nq) * D
                                               : vrow + (r - nq - p.Hkv) * D;
        a[e][0] = *reinterpret_cast<const uint4*>(src);
        a[e][1] = *reinterpret_cast<const uint4*>(src + D / 2);
      }
    }
  };
  const bool early = l < p.L && (!RING || (!p.count && t >= p.T - p.W));
  if (early) load(first, min(first + per, (all + P::kRows - 1) / P::kRows), all);
  const int n = count < 0 ? 0 : count < p.T ? static_cast<int>(count) : p.T;
  const bool live = l < p.L && t < n && !(RING && pos < 0);
  unsigned long long ticket = 0, tickets = 0;
  if (RING) {
    // The sequence's L n tokens, `parts` warps each, are counted where all threads of a CTA have read pos (and used it);
    // the CTA that completes the count advances it, in the end: the answer takes a trip to L2.
    tickets = static_cast<unsigned long long>(__syncthreads_count(live && lane == 0));
    if (threadIdx.x == 0 && tickets != 0) ticket = atomicAdd(p.tickets + b, tickets);
    if (threadIdx.x == 0 && blockIdx.x == 0 && pos < 0) atomicOr(p.status, CMC_DEVFLAG_BAD_POS);
  }
  if (live) {
    const bool rope = p.prep.rope != 0, norm = p.prep.q_weight || p.prep.k_weight;
    const unsigned long long at = static_cast<unsigned long long>(p.prep.rope_offset + pos + t) +
                                  static_cast<unsigned long long>(moved);
    if (rope || norm) {
#pragma unroll
      for (int e = 0; e < D / 64; ++e) {
        const int i = lane + 32 * e;
        const float2 cs = rope ? rope_cos_sin(at, turns[e]) : make_float2(1.f, 0.f);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float* w = x == 0 ? p.prep.q_weight : p.prep.k_weight;
          const float g = w ? w[static_cast<long long>(l) * D + i] : 1.f, h = w ? w[static_cast<long long>(l) * D + D / 2 + i] : 1.f;
          table.pair[x][i % 8][i / 8] = pair_factors(g, h, cs);
        }
      }
      __syncwarp();
    }
    // Rows of k and v that the ring does not keep are left out.
    const bool kept = !RING || t >= n - p.W;
    long long slot = 0;
    if (RING && kept) {
      const unsigned long long at = static_cast<unsigned long long>(pos) + static_cast<unsigned long long>(t);
      slot = (at >> 32) == 0 ? static_cast<unsigned>(at) % static_cast<unsigned>(p.W)
                             : static_cast<long long>(at % static_cast<unsigned>(p.W));
    }
    const int rows = kept ? all : nq;
    const int end = min(first + per, (rows + P::kRows - 1) / P::kRows);
    const long long unit0 = (static_cast<long long>(b) * p.L + l) * p.Hkv;
    uint16_t* to_q = p.out_q + row0 * p.Hq * D + 8 * c;
    uint16_t* to_k = RING ? p.ring_k + (unit0 * p.W + slot) * D + 8 * c : p.out_k + row0 * p.Hkv * D + 8 * c;
    uint16_t* to_v = p.ring_v + (unit0 * p.W + slot) * D + 8 * c;
    const long long step = RING ? static_cast<long long>(p.W) * D : D;  // from one KV head's row to the next
    auto store = [&](int r, const uint4 (&x)[2]) {
      const bool is_v = r >= nq + p.Hkv;
      uint16_t* dst = r < nq    ? to_q + r * D
                      : is_v ? to_v + (r - nq - p.Hkv) * step
                             : to_k + (r - nq) * step;
      *reinterpret_cast<uint4*>(dst) = x[0];
      *reinterpret_cast<uint4*>(dst + D / 2) = x[1];
      if (RING && is_v && c == 0 && p.ring_weight) p.ring_weight[(unit0 + r - nq - p.Hkv) * p.W + slot] = 0.f;
    };
    uint32_t odd = 0;  // the most that a row's mean, as a place among floats, is above kOddMean (modulo 2^32: or below)
    for (int s0 = first; s0 < end; s0 += kPrefillBatch) {
      if (s0 > first || !early) load(s0, end, rows);
#pragma unroll
      for (int e = 0; e < kPrefillBatch; ++e) {
        if (s0 + e >= end) break;
        const int r = (s0 + e) * P::kRows + sub;
        const bool is_v = r >= nq + p.Hkv;
        const bool is_q = r < nq;
        float f = 1.f;
        if (norm) {
          const bool plain = is_v || (is_q ? p.prep.q_weight : p.prep.k_weight) == nullptr;
          const float mean = row_mean<D>(prep_squares<D>(a[e][0], a[e][1], 1.f), p.prep.eps);
          f = rsqrtf(mean);
          if (PLACE) {  // at once, since the row is not there any more later
            const bool mine = !plain && odd_mean(mean);
            if (__any_sync(0xffffffffu, mine)) {
              uint4 x[2] = {a[e][0], a[e][1]};
              const float g = prep_odd_row<D>(x, mean, p.prep.eps);
              if (mine) {
                f = g;
                a[e][0] = x[0];
                a[e][1] = x[1];
              }
            }
          } else {
            odd = __viaddmax_u32(__float_as_uint(mean), 0u - kOddMean, odd);
          }
          if (plain) f = 1.f;
        }
        if ((rope || norm) && !is_v) prep_chunks<D>(a[e], f, rope, table.pair[is_q ? 0 : 1], c);
        if (r < rows) store(r, a[e]);
      }
    }
    if (!PLACE && __any_sync(0xffffffffu, odd >= kOddMeans)) {  // some row's mean is odd: those that have a norm again
#pragma unroll 1
      for (int s0 = first; s0 < end; ++s0) {
        load(s0, s0 + 1, rows);
        const int r = s0 * P::kRows + sub;
        const bool has = r < min(rows, nq + p.Hkv) && (r < nq ? p.prep.q_weight : p.prep.k_weight) != nullptr;
        const float mean = row_mean<D>(prep_squares<D>(a[0][0], a[0][1], 1.f), p.prep.eps);
        const float f = prep_odd_row<D>(a[0], mean, p.prep.eps);
        prep_chunks<D>(a[0], f, rope, table.pair[r < nq ? 0 : 1], c);
        if (has && odd_mean(mean)) store(r, a[0]);
      }
    }
  }
  if (RING && threadIdx.x == 0 && tickets != 0 &&
      ticket + tickets == static_cast<unsigned long long>(p.L) * static_cast<unsigned>(n) * static_cast<unsigned>(p.parts)) {
    p.pos[b] = pos + n;
    p.tickets[b] = 0ull;
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
  // Warps read and write in any order: an output meets no input, but for heads prepared where they are, and no other output.
  const long long tokens = items * m.B;
  auto heads = [&](const void* a, long long stride, long long row) { return Range{a, static_cast<size_t>((tokens - 1) * stride + row) * 2}; };
  const size_t ring_bytes = static_cast<size_t>(m.B) * m.L * m.Hkv * m.W * m.d * 2;
  const Range in[] = {heads(q, q_stride, qd), heads(k, k_stride, kd), heads(v, v_stride, kd)};
  const Range outs[] = {heads(out_q, qd, qd), heads(out_k, kd, kd), {ring_k, ring_bytes}, {ring_v, ring_bytes}};
  for (int o = 0; o < 4; ++o) {
    for (int i = 0; i < 3; ++i) {
      const bool there = i == o && o < 2 && same(in[i], outs[o]);  // out_q in q, out_k in k
      if (!there && meet(outs[o], in[i])) return CMC_ERR_RANGE;
    }
    for (int i = 0; i < o; ++i)
      if (meet(outs[o], outs[i])) return CMC_ERR_RANGE;
  }
  PrefillParams p;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  st = prep_params(prep, m.d, s, &p.prep);
  if (st != CMC_OK) return st;
  // Nor do the weights, the positions and the workspace meet anything, or the outputs what the preparation reads.
  const size_t each = static_cast<size_t>(m.B) * 8, gains = static_cast<size_t>(m.L) * m.d * 4;
  const Range more_in[] = {{count, each}, {p.prep.evicted, each}, {p.prep.q_weight, gains}, {p.prep.k_weight, gains}, {ring ? nullptr : pos, each}};
  const Range more_outs[] = {{ring_weight, ring_bytes / (2 * m.d) * 4}, {ring ? pos : nullptr, each}, {workspace, ring ? ws_partials_off(m.B) : 0}};
  if (any_meet(outs, more_in) || any_meet(more_outs, in) || any_meet(more_outs, outs) || any_meet(more_outs, more_in) || any_meet(more_outs))
    return CMC_ERR_RANGE;
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
  const bool place = (q && q == out_q) || k == out_k;
  auto kern = ring ? (place ? (m.d == 128 ? prefill_kernel<128, true, true> : prefill_kernel<64, true, true>)
                            : (m.d == 128 ? prefill_kernel<128, true, false> : prefill_kernel<64, true, false>))
                   : (place ? (m.d == 128 ? prefill_kernel<128, false, true> : prefill_kernel<64, false, true>)
                            : (m.d == 128 ? prefill_kernel<128, false, false> : prefill_kernel<64, false, false>));
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
