// Decode attention over [Tier-1 | Tier-2] that adds to each key's weight the probabilities it gets
// (cmc_two_tier_decode_attn_weighted), and the decode step around it (cmc_decode_step_weighted):
//   out[h]    = sum_j p_hj v_j,   p_hj = 2^(s_hj - M_h) / l_h,   s = scale log2(e) q_h . k_j
//   weight[j] += sum of p_hj over the G query heads of the KV head
// The probabilities need the final maximum M and sum l, which one pass over the keys knows only at its
// end.  So each CTA keeps the products q . k of its keys in shared memory (4 G bytes a key, beside the key's 4 d bytes
// in HBM), and when its unit's M and l are known goes over them once more.
//
// Bound: HBM, 4 d + 8 bytes a key against 4 G d flops.  A unit (sequence, layer, KV head) is taken by a CTA of
// eight warps or a cluster of up to eight CTAs; its keys are cut into blocks of 16, ceil(k / 16) of Tier-1, then those of
// the ring's occupied slots, and warp w of the unit's 8 cm takes blocks w, w + 8 cm, ...
//
// K and V go from HBM straight to the registers that feed the products: no stage in shared memory, no
// barrier, and rows that hold no key are simply not read.  With the products of cmc_attn.cu,
//   S^T = K Q^T     16 keys as the M rows, the G query heads (padded to 8) as the columns
//   O^T += V^T P^T  16 rows of the head dimension, the heads, the 16 keys as the k-step
// (mma.sync m16n8k16; 4 flops a byte: the tensor pipe is all but idle), the order of d within the first and of the
// M rows of the second is free, and chosen so that 16-byte loads fill the fragments:
//   K: lane (g, t) = (lane / 4, lane % 4) has chunk 4 i + t (elements 32 i + 8 t ..) of rows g and g + 8; its four words are
//      the k pairs of steps 2 i and 2 i + 1, and Q's fragments are the same chunks of row g of Q.
//   V: lane (g, t) has chunk 8 h + g of rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9; words of two rows make pairs of keys (prmt), and
//      row g / g + 8 of product 4 h + w is column 64 h + 8 g + 2 w / + 1.
// The next block's K is requested when S^T has taken this one's, its V when O^T has.
//
// The new token (fused step) is read from k_new and v_new where its slot's row would be, by the warp that has
// the block, which stores it to the ring as well.  With norm or rotary embedding two warps first
// prepare q and the new key; q is then held as the sum of two bf16 (products off by 2^-17 of a term: the
// probabilities are sums in fp32 that outlive the call), the key rounded to bf16 as it is stored.
#include <algorithm>
#include <atomic>

#include "cmc_prep.cuh"

namespace cmc {

constexpr int kWWarps = 8;
constexpr int kWThreads = 32 * kWWarps;
constexpr int kBlkKeys = 16;
// Products that a CTA keeps in shared memory, in bytes; two CTAs share an SM at that.  Units too long for a cluster of
// eight at that keep them in the workspace.
constexpr int kScoreBytes = 73728;

struct WeightedParams {
  const uint16_t* q;      // [B, L, Hq, d]
  const uint16_t* t1k;    // [B, L, Hkv, N, d]
  const uint16_t* t1v;
  float* t1w;             // [B, L, Hkv, N]
  uint16_t* ring_k;       // [B, L, Hkv, W, d]
  uint16_t* ring_v;
  float* ring_w;          // [B, L, Hkv, W]
  int64_t* pos;           // [B]
  const uint16_t* k_new;  // [B, L, Hkv, d]
  const uint16_t* v_new;
  uint16_t* out;          // [B, L, Hq, d]
  uint32_t* status;
  unsigned long long* tickets;
  float* scratch;         // products of a unit too long for shared memory, or NULL
  int L, Hkv, N, k, W, LH;
  int cm;                 // CTAs per unit
  int nb1;                // blocks of Tier-1
  int iters;              // blocks a warp takes at most
  int prefetch;           // blocks per warp prefetched into L2 before the grid dependency wait
  float scale_log2;
  PrepParams prep;
};

__host__ __device__ constexpr int wrow_floats(int D) { return D + 4; }

// Shared memory: Q as bf16 sums and the prepared key (with PREP), the warps' states, a cluster's record, then
// the products.
template <int D, int G, bool PREP>
struct WSmem {
  static constexpr int kQ = 0;                                     // [2][8][D] bf16: high and low parts
  static constexpr int kNew = kQ + (PREP ? 2 * 8 * D * 2 : 0);     // [D] bf16
  static constexpr int kTab = kNew + (PREP ? D * 2 : 0);           // [2][D / 2] (cos, sin)
  static constexpr int kM = kTab + (PREP ? 2 * D * 4 : 0);         // [warp][8] maxima, [warp][8] sums
  static constexpr int kO = kM + kWWarps * 16 * 4;                 // [warp][G][wrow_floats(D)]
  static constexpr int kRec = kO + kWWarps * G * wrow_floats(D) * 4;  // [G][D] output, [8][2] maximum and sum
  static constexpr int kFin = kRec + (G * D + 16) * 4;             // [8] final maxima, [8] 1 / sums
  static constexpr int kScores = kFin + 16 * 4;
  static_assert(kScores % 16 == 0, "read by 16 bytes");
};

__device__ __forceinline__ void wmma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                     uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A 16-byte load of what a launch reads once.
__device__ __forceinline__ uint4 ld_once(const uint16_t* p, uint64_t policy) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;\n"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p), "l"(policy)
               : "memory");
  return r;
}

__device__ __forceinline__ float ld_peer_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_peer_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];\n"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}

// A block of a unit: its rows in memory and how many hold keys.
struct Blk {
  const uint16_t* k;
  const uint16_t* v;
  int rows;     // 1 .. 16
  int new_row;  // the new token's, or -1
};

template <int D>
__device__ __forceinline__ Blk blk_of(const WeightedParams& p, long long u, int blk, int count, int new_slot) {
  Blk r;
  r.new_row = -1;
  if (blk < p.nb1) {
    const long long e = (u * p.N + blk * kBlkKeys) * D;
    r.k = p.t1k + e;
    r.v = p.t1v + e;
    r.rows = min(p.k - blk * kBlkKeys, kBlkKeys);
  } else {
    const int s0 = (blk - p.nb1) * kBlkKeys;
    const long long e = (u * p.W + s0) * D;
    r.k = p.ring_k + e;
    r.v = p.ring_v + e;
    r.rows = min(count - s0, kBlkKeys);
    if (new_slot >= s0 && new_slot < s0 + kBlkKeys) r.new_row = new_slot - s0;
  }
  return r;
}

// K of a block: chunks 4 i + t of rows g and g + 8.  `newk`: the new token's row.
template <int D>
__device__ __forceinline__ void load_k(const Blk& b, const uint16_t* newk, uint16_t* to, int g, int t,
                                       uint64_t pol, uint4 (&kr)[2][D / 32]) {
  if (b.rows == kBlkKeys && b.new_row < 0) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) kr[h][i] = ld_once(b.k + (g + 8 * h) * D + 32 * i + 8 * t, pol);
    return;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = g + 8 * h;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const int c = 32 * i + 8 * t;
      kr[h][i] = make_uint4(0u, 0u, 0u, 0u);
      if (row == b.new_row) {
        kr[h][i] = *reinterpret_cast<const uint4*>(newk + c);
        *reinterpret_cast<uint4*>(to + c) = kr[h][i];
      } else if (row < b.rows) {
        kr[h][i] = ld_once(b.k + row * D + c, pol);
      }
    }
  }
}

// V of a block: chunks 8 h + g of rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9.
template <int D>
__device__ __forceinline__ void load_v(const Blk& b, const uint16_t* newv, uint16_t* to, int g, int t,
                                       uint64_t pol, uint4 (&vr)[4][D / 64]) {
  if (b.rows == kBlkKeys && b.new_row < 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < D / 64; ++h)
        vr[j][h] = ld_once(b.v + (2 * t + (j & 1) + 8 * (j >> 1)) * D + 64 * h + 8 * g, pol);
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int row = 2 * t + (j & 1) + 8 * (j >> 1);
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
      const int c = 64 * h + 8 * g;
      vr[j][h] = make_uint4(0u, 0u, 0u, 0u);
      if (row == b.new_row) {
        vr[j][h] = *reinterpret_cast<const uint4*>(newv + c);
        *reinterpret_cast<uint4*>(to + c) = vr[j][h];
      } else if (row < b.rows) {
        vr[j][h] = ld_once(b.v + row * D + c, pol);
      }
    }
  }
}

// Norm and rotation of the unit's G query heads (warp 0, and of the new key's row warp 1), into shared memory.
template <int D, int G>
__device__ __forceinline__ void prepare(const WeightedParams& p, long long u, int b, long long pos, int warp,
                                        int lane, uint8_t* smem) {
  using S = WSmem<D, G, true>;
  using P = Prep<D>;
  const int c = lane % P::kLanes, sub = lane / P::kLanes;
  const int l = static_cast<int>(u / p.Hkv % p.L);
  const float* w = warp == 0 ? p.prep.q_weight : p.prep.k_weight;
  if (w) w += static_cast<long long>(l) * D;
  float2 cs[8];
  if (p.prep.rope) {
    unsigned long long at = static_cast<unsigned long long>(p.prep.rope_offset + pos);
    if (p.prep.evicted) at += static_cast<unsigned long long>(p.prep.evicted[b]);
    float2* tab = reinterpret_cast<float2*>(smem + S::kTab) + warp * (D / 2);
    prep_table<D>(p.prep, at, lane, tab);
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = tab[8 * c + e];
  }
  const int rows = warp == 0 ? 8 : 1;
  const uint16_t* src = warp == 0 ? p.q + u * G * D : p.k_new + u * D;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += P::kRows) {
    const int r = r0 + sub;
    uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
    if (r < (warp == 0 ? G : 1)) {
      lo = *reinterpret_cast<const uint4*>(src + r * D + 8 * c);
      hi = *reinterpret_cast<const uint4*>(src + r * D + D / 2 + 8 * c);
    }
    float x[16];
    prep_unpack(lo, hi, x);
    prep_norm<D>(x, w, p.prep.eps, c);
    if (p.prep.rope) prep_rotate(x, cs);
    const uint4 a = prep_pack(x), z = prep_pack(x + 8);
    if (warp == 1) {
      if (r < 1) {
        uint16_t* to = reinterpret_cast<uint16_t*>(smem + S::kNew);
        *reinterpret_cast<uint4*>(to + 8 * c) = a;
        *reinterpret_cast<uint4*>(to + D / 2 + 8 * c) = z;
      }
    } else if (r < 8) {
      uint16_t* to = reinterpret_cast<uint16_t*>(smem + S::kQ) + r * D;
      *reinterpret_cast<uint4*>(to + 8 * c) = a;
      *reinterpret_cast<uint4*>(to + D / 2 + 8 * c) = z;
      float ah[8], zh[8];
      unpack8(a, ah);
      unpack8(z, zh);
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // what is left (nothing that can be held where the high part is infinite)
        x[e] = fabsf(ah[e]) < INFINITY ? x[e] - ah[e] : 0.f;
        x[8 + e] = fabsf(zh[e]) < INFINITY ? x[8 + e] - zh[e] : 0.f;
      }
      to += 8 * D;
      *reinterpret_cast<uint4*>(to + 8 * c) = prep_pack(x);
      *reinterpret_cast<uint4*>(to + D / 2 + 8 * c) = prep_pack(x + 8);
    }
  }
}

template <int D, int G, bool FUSED, bool PREP>
__global__ void __launch_bounds__(kWThreads, 2)
weighted_attn_kernel(const __grid_constant__ WeightedParams p) {
  using S = WSmem<D, G, PREP>;
  constexpr int DP = wrow_floats(D);
  constexpr int KC = D / 32;  // K chunks of a lane and row
  constexpr int VH = D / 64;  // V chunks of a lane and row
  extern __shared__ __align__(16) uint8_t smem[];
  float* merge_m = reinterpret_cast<float*>(smem + S::kM);
  float* merge_l = merge_m + kWWarps * 8;
  float* merge_o = reinterpret_cast<float*>(smem + S::kO);
  float* rec_o = reinterpret_cast<float*>(smem + S::kRec);
  float* rec_ml = rec_o + G * D;
  float* fin_m = reinterpret_cast<float*>(smem + S::kFin);
  float* fin_r = fin_m + 8;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  const long long u = blockIdx.x / static_cast<unsigned>(p.cm);
  const int rank = static_cast<int>(blockIdx.x - u * p.cm);
  const int b = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(p.LH));
  const int stride = p.cm * kWWarps;
  const int first = rank * kWWarps + warp;

  // The warp's first blocks, into L2: hints, which may come before the wait.
  if (lane < 2 * p.prefetch) {
    const int blk = first + (lane >> 1) * stride;
    const uint16_t* base = nullptr;
    int rows = 0;
    if (blk < p.nb1) {
      base = ((lane & 1) ? p.t1v : p.t1k) + (u * p.N + blk * kBlkKeys) * D;
      rows = min(p.k - blk * kBlkKeys, kBlkKeys);
    } else if ((blk - p.nb1) * kBlkKeys < p.W) {
      base = ((lane & 1) ? p.ring_v : p.ring_k) + (u * p.W + (blk - p.nb1) * kBlkKeys) * D;
      rows = min(p.W - (blk - p.nb1) * kBlkKeys, kBlkKeys);
    }
    if (rows > 0)
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(base), "r"(rows * D * 2) : "memory");
  }
  pdl_wait();
  pdl_trigger();

  long long pos;
  asm volatile("ld.global.cg.s64 %0, [%1];\n" : "=l"(pos) : "l"(p.pos + b) : "memory");
  const uint16_t* newk = FUSED ? p.k_new + u * D : nullptr;
  const uint16_t* newv = FUSED ? p.v_new + u * D : nullptr;
  uint4 qa[KC];
#pragma unroll
  for (int i = 0; i < KC; ++i) {
    qa[i] = make_uint4(0u, 0u, 0u, 0u);
    if (!PREP && g < G) qa[i] = *reinterpret_cast<const uint4*>(p.q + (u * G + g) * D + 32 * i + 8 * t);
  }
  const bool bad = pos < 0;
  int count = 0, new_slot = -1;
  if (!bad) {
    if (FUSED) {
      count = static_cast<int>(pos + 1 < p.W ? pos + 1 : p.W);
      new_slot = (pos >> 32) == 0
                     ? static_cast<int>(static_cast<unsigned>(pos) % static_cast<unsigned>(p.W))
                     : static_cast<int>(pos % p.W);
    } else {
      count = static_cast<int>(pos < p.W ? pos : p.W);
    }
  }
  const int nblk = bad ? 0 : p.nb1 + (count + kBlkKeys - 1) / kBlkKeys;
  if (PREP) {
    newk = reinterpret_cast<const uint16_t*>(smem + S::kNew);
    if (warp < 2) prepare<D, G>(p, u, b, pos, warp, lane, smem);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KC; ++i)
      qa[i] = *reinterpret_cast<const uint4*>(smem + S::kQ + (g * D + 32 * i + 8 * t) * 2);
  }
  uint16_t* put_k = p.ring_k + (u * p.W + new_slot) * D;  // (not used without a new token)
  uint16_t* put_v = p.ring_v + (u * p.W + new_slot) * D;

  // The products of this CTA's keys: [iteration][warp][16 keys][G].
  float* scores = p.scratch ? p.scratch + static_cast<long long>(blockIdx.x) * p.iters * kWWarps * kBlkKeys * G
                            : reinterpret_cast<float*>(smem + S::kScores);

  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
  float o[4 * VH][4];
#pragma unroll
  for (int j = 0; j < 4 * VH; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
  uint4 kr[2][KC], vr[4][VH];
  const uint64_t pol = policy_evict_first();
  int blk = first;
  Blk cur;
  if (blk < nblk) {
    cur = blk_of<D>(p, u, blk, count, new_slot);
    load_k<D>(cur, newk, put_k, g, t, pol, kr);
    load_v<D>(cur, newv, put_v, g, t, pol, vr);
  }
  float* sc = scores + (warp * kBlkKeys + g) * G + 2 * t;
  while (blk < nblk) {
    float sa[2][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) sa[0][e] = sa[1][e] = 0.f;
#pragma unroll
    for (int i = 0; i < KC; ++i) {
      wmma(sa[0], kr[0][i].x, kr[1][i].x, kr[0][i].y, kr[1][i].y, qa[i].x, qa[i].y);
      wmma(sa[1], kr[0][i].z, kr[1][i].z, kr[0][i].w, kr[1][i].w, qa[i].z, qa[i].w);
    }
    if (PREP) {
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        const uint4 ql = *reinterpret_cast<const uint4*>(smem + S::kQ + ((8 + g) * D + 32 * i + 8 * t) * 2);
        wmma(sa[0], kr[0][i].x, kr[1][i].x, kr[0][i].y, kr[1][i].y, ql.x, ql.y);
        wmma(sa[1], kr[0][i].z, kr[1][i].z, kr[0][i].w, kr[1][i].w, ql.z, ql.w);
      }
    }
    const int rows = cur.rows;
    const int next = blk + stride;
    Blk nb;
    if (next < nblk) {
      nb = blk_of<D>(p, u, next, count, new_slot);
      load_k<D>(nb, newk, put_k, g, t, pol, kr);
    }
    float v[4];  // keys g (0, 1) and g + 8 (2, 3), heads 2 t and 2 t + 1
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = sa[0][e] + sa[1][e];
    if (g >= rows) v[0] = v[1] = -INFINITY;
    if (g + 8 >= rows) v[2] = v[3] = -INFINITY;
    if (2 * t < G) {
      if (G == 1) {
        sc[0] = v[0];
        sc[8] = v[2];
      } else {
        *reinterpret_cast<float2*>(sc) = make_float2(v[0], v[1]);
        *reinterpret_cast<float2*>(sc + 8 * G) = make_float2(v[2], v[3]);
      }
    }
    sc += kWWarps * kBlkKeys * G;
    float mx0 = fmaxf(v[0], v[2]), mx1 = fmaxf(v[1], v[3]);
#pragma unroll
    for (int off = 4; off < 32; off <<= 1) {
      mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, off));
      mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, off));
    }
    mx0 *= p.scale_log2;
    mx1 *= p.scale_log2;
    const bool up0 = mx0 > m_run[0], up1 = mx1 > m_run[1];
    if (__any_sync(0xffffffffu, up0 || up1)) {
      const float alpha0 = up0 ? ex2(m_run[0] - mx0) : 1.f;
      const float alpha1 = up1 ? ex2(m_run[1] - mx1) : 1.f;
      if (up0) m_run[0] = mx0;
      if (up1) m_run[1] = mx1;
      l_run[0] *= alpha0;
      l_run[1] *= alpha1;
#pragma unroll
      for (int j = 0; j < 4 * VH; ++j) {
        o[j][0] *= alpha0;
        o[j][1] *= alpha1;
        o[j][2] *= alpha0;
        o[j][3] *= alpha1;
      }
    }
    float pr[4] = {0.f, 0.f, 0.f, 0.f};
    if (m_run[0] != -INFINITY) {
      pr[0] = ex2(fmaf(v[0], p.scale_log2, -m_run[0]));
      pr[2] = ex2(fmaf(v[2], p.scale_log2, -m_run[0]));
    }
    if (m_run[1] != -INFINITY) {
      pr[1] = ex2(fmaf(v[1], p.scale_log2, -m_run[1]));
      pr[3] = ex2(fmaf(v[3], p.scale_log2, -m_run[1]));
    }
    l_run[0] += pr[0] + pr[2];
    l_run[1] += pr[1] + pr[3];
    // P^T as the B operand: packed to bf16 (outputs are bf16; the sums are not rounded) and transposed
    const uint32_t pb0 = movmatrix_trans(pack_bf16_rn(pr[0], pr[1]));
    const uint32_t pb1 = movmatrix_trans(pack_bf16_rn(pr[2], pr[3]));
#pragma unroll
    for (int h = 0; h < VH; ++h) {
      const uint32_t* r0 = reinterpret_cast<const uint32_t*>(&vr[0][h]);
      const uint32_t* r1 = reinterpret_cast<const uint32_t*>(&vr[1][h]);
      const uint32_t* r2 = reinterpret_cast<const uint32_t*>(&vr[2][h]);
      const uint32_t* r3 = reinterpret_cast<const uint32_t*>(&vr[3][h]);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        wmma(o[4 * h + w], __byte_perm(r0[w], r1[w], 0x5410), __byte_perm(r0[w], r1[w], 0x7632),
             __byte_perm(r2[w], r3[w], 0x5410), __byte_perm(r2[w], r3[w], 0x7632), pb0, pb1);
    }
    if (next < nblk) {
      load_v<D>(nb, newv, put_v, g, t, pol, vr);
      cur = nb;
    }
    blk = next;
  }

  // ---- the warps' states ----
#pragma unroll
  for (int off = 4; off < 32; off <<= 1) {
    l_run[0] += __shfl_xor_sync(0xffffffffu, l_run[0], off);
    l_run[1] += __shfl_xor_sync(0xffffffffu, l_run[1], off);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int hh = 2 * t + e;
    if (hh < G) {
      float* ow = merge_o + (warp * G + hh) * DP + 8 * g;
#pragma unroll
      for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int w = 0; w < 4; ++w)
          *reinterpret_cast<float2*>(ow + 64 * h + 2 * w) = make_float2(o[4 * h + w][e], o[4 * h + w][2 + e]);
      if (g == 0) {
        merge_m[warp * 8 + hh] = m_run[e];
        merge_l[warp * 8 + hh] = l_run[e];
      }
    }
  }

  // This CTA's keys once more: key x of its iterations' blocks.  The first weights are requested
  // before the merge.
  const int mine = nblk > rank * kWWarps ? (nblk - rank * kWWarps + stride - 1) / stride : 0;  // iterations
  const int nkeys = mine * kWWarps * kBlkKeys;
  auto weight_of = [&](int x) -> float* {
    const int w = (x / kBlkKeys) % kWWarps;
    const int bk = rank * kWWarps + w + x / (kBlkKeys * kWWarps) * stride;
    const int r = x % kBlkKeys;
    if (bk < p.nb1) return bk * kBlkKeys + r < p.k ? p.t1w + u * p.N + bk * kBlkKeys + r : nullptr;
    const int s = (bk - p.nb1) * kBlkKeys + r;
    return bk < nblk && s < count ? p.ring_w + u * p.W + s : nullptr;
  };
  const float* fresh = FUSED && new_slot >= 0 ? p.ring_w + u * p.W + new_slot : nullptr;
  constexpr int kAhead = 4;
  float* wp[kAhead];
  float wv[kAhead];
#pragma unroll
  for (int e = 0; e < kAhead; ++e) {
    const int x = tid + e * kWThreads;
    wp[e] = x < nkeys ? weight_of(x) : nullptr;
    wv[e] = wp[e] && wp[e] != fresh ? *wp[e] : 0.f;
  }
  __syncthreads();
  if (FUSED && tid == 0) {
    // every thread of the CTA has read pos; the last CTA of the sequence to come here advances it
    __threadfence();
    if (atomicAdd(p.tickets + b, 1ull) + 1 == static_cast<unsigned long long>(p.LH) * p.cm) {
      if (!bad) p.pos[b] = pos + 1;
      p.tickets[b] = 0ull;
    }
  }
  if (bad && tid == 0 && rank == 0) atomicOr(p.status, CMC_DEVFLAG_BAD_POS);

  // ---- merge: four columns of one head a thread, the warps in order ----
  constexpr int NGR = G * D / 4;
  const long long out_base = u * (G * D);
  for (int x = tid; x < NGR; x += kWThreads) {
    const int hh = (4 * x) / D, c = (4 * x) % D;
    float M = merge_m[hh];
#pragma unroll
    for (int w = 1; w < kWWarps; ++w) M = fmaxf(M, merge_m[w * 8 + hh]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float Ls = 0.f;
    if (M != -INFINITY) {
#pragma unroll
      for (int w = 0; w < kWWarps; ++w) {
        const float f = ex2(merge_m[w * 8 + hh] - M);
        const float4 y = *reinterpret_cast<const float4*>(merge_o + (w * G + hh) * DP + c);
        acc.x = fmaf(f, y.x, acc.x);
        acc.y = fmaf(f, y.y, acc.y);
        acc.z = fmaf(f, y.z, acc.z);
        acc.w = fmaf(f, y.w, acc.w);
        Ls = fmaf(f, merge_l[w * 8 + hh], Ls);
      }
    }
    if (p.cm == 1) {
      const float inv = Ls == 0.f ? 0.f : 1.f / Ls;
      *reinterpret_cast<uint2*>(p.out + out_base + hh * D + c) =
          make_uint2(pack_bf16_rn(acc.x * inv, acc.y * inv), pack_bf16_rn(acc.z * inv, acc.w * inv));
      if (c == 0) {
        fin_m[hh] = M;
        fin_r[hh] = inv;
      }
    } else {
      *reinterpret_cast<float4*>(rec_o + hh * D + c) = acc;
      if (c == 0) {
        rec_ml[2 * hh] = M;
        rec_ml[2 * hh + 1] = Ls;
      }
    }
  }
  if (p.cm > 1) {
    // Each CTA of the cluster merges its share of the columns from its peers' records.
    cluster_sync_all();
    const uint32_t o_a = smem_addr(rec_o), ml_a = smem_addr(rec_ml);
    const int SL = (NGR + p.cm - 1) / p.cm;
    const int x1 = min((rank + 1) * SL, NGR);
    auto merged = [&](int hh, float& M, float& Ls) {
      M = -INFINITY;
      Ls = 0.f;
      for (int r = 0; r < p.cm; ++r) M = fmaxf(M, ld_peer_f32(peer_smem(ml_a + 8 * hh, r)));
      if (M == -INFINITY) return;
      for (int r = 0; r < p.cm; ++r)
        Ls = fmaf(ex2(ld_peer_f32(peer_smem(ml_a + 8 * hh, r)) - M), ld_peer_f32(peer_smem(ml_a + 8 * hh + 4, r)), Ls);
    };
    for (int x = rank * SL + tid; x < x1; x += kWThreads) {
      const int hh = (4 * x) / D, c = (4 * x) % D;
      float M, Ls;
      merged(hh, M, Ls);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      if (M != -INFINITY) {
        for (int r = 0; r < p.cm; ++r) {
          const float f = ex2(ld_peer_f32(peer_smem(ml_a + 8 * hh, r)) - M);
          const float4 y = ld_peer_f4(peer_smem(o_a + (hh * D + c) * 4, r));
          acc.x = fmaf(f, y.x, acc.x);
          acc.y = fmaf(f, y.y, acc.y);
          acc.z = fmaf(f, y.z, acc.z);
          acc.w = fmaf(f, y.w, acc.w);
        }
      }
      const float inv = Ls == 0.f ? 0.f : 1.f / Ls;
      *reinterpret_cast<uint2*>(p.out + out_base + hh * D + c) =
          make_uint2(pack_bf16_rn(acc.x * inv, acc.y * inv), pack_bf16_rn(acc.z * inv, acc.w * inv));
    }
    if (tid >= kWThreads - G) {  // the heads' final maxima and sums, for the weights
      const int hh = tid - (kWThreads - G);
      float M, Ls;
      merged(hh, M, Ls);
      fin_m[hh] = M;
      fin_r[hh] = Ls == 0.f ? 0.f : 1.f / Ls;
    }
    cluster_arrive();  // this thread reads its peers' memory no more
  }
  __syncthreads();

  // ---- the weights ----
  float M[G], R[G];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    M[h] = fin_m[h];
    R[h] = fin_r[h];
  }
  for (int x0 = tid; x0 < nkeys; x0 += kAhead * kWThreads) {
    if (x0 != tid) {
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const int x = x0 + e * kWThreads;
        wp[e] = x < nkeys ? weight_of(x) : nullptr;
        wv[e] = wp[e] && wp[e] != fresh ? *wp[e] : 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      if (!wp[e]) continue;
      const float* s = scores + static_cast<long long>(x0 + e * kWThreads) * G;
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < G; ++h) sum = fmaf(ex2(fmaf(s[h], p.scale_log2, -M[h])), R[h], sum);
      *wp[e] = wv[e] + sum;
    }
  }
  if (p.cm > 1) cluster_wait();  // no peer reads this CTA's memory any more
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// Blocks that a warp of a cluster of cm CTAs takes at most.
static int iters_of(const cmc_dims& m, int cm) {
  const long long nblk = (static_cast<long long>(m.k) + kBlkKeys - 1) / kBlkKeys +
                         (static_cast<long long>(m.W) + kBlkKeys - 1) / kBlkKeys;
  return static_cast<int>((nblk + cm * kWWarps - 1) / (cm * kWWarps));
}
static size_t score_bytes(const cmc_dims& m, int cm) {
  return static_cast<size_t>(iters_of(m, cm)) * kWWarps * kBlkKeys * (m.Hq / m.Hkv) * 4;
}
static bool needs_scratch(const cmc_dims& m) { return score_bytes(m, kMaxClusterCtas) > kScoreBytes; }
static size_t weighted_ws(const cmc_dims& m) {
  const size_t units = static_cast<size_t>(m.B) * m.L * m.Hkv;
  return ws_partials_off(m.B) + (needs_scratch(m) ? units * kMaxClusterCtas * score_bytes(m, kMaxClusterCtas) : 0);
}

// CTAs per unit: as many as it takes to fill the device, at most one per eight blocks; more where the unit's
// products would not go into shared memory.
static int plan_cm(const cmc_dims& m, int per_sm) {
  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  long long cm = static_cast<long long>(per_sm) * sm_count() / units;
  const long long nblk = (static_cast<long long>(m.k) + kBlkKeys - 1) / kBlkKeys +
                         (static_cast<long long>(m.W) + kBlkKeys - 1) / kBlkKeys;
  cm = std::min(cm, (nblk + kWWarps - 1) / kWWarps);
  cm = std::max(1LL, std::min<long long>(cm, kMaxClusterCtas));
  while (cm < kMaxClusterCtas && score_bytes(m, static_cast<int>(cm)) > kScoreBytes) ++cm;
  return static_cast<int>(cm);
}

template <int D, int G, bool FUSED, bool PREP>
static int per_sm_of(int* out) {
  constexpr int smem = WSmem<D, G, PREP>::kScores + kScoreBytes;
  auto kern = weighted_attn_kernel<D, G, FUSED, PREP>;
  static std::atomic<int> known[64];
  int dev = 0;
  int st = record_cuda_error(cudaGetDevice(&dev));
  if (st != CMC_OK) return st;
  int per_sm = (dev >= 0 && dev < 64) ? known[dev].load(std::memory_order_acquire) : 0;
  if (per_sm <= 0) {
    st = record_cuda_error(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (st != CMC_OK) return st;
    st = record_cuda_error(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, kWThreads, smem));
    if (st != CMC_OK) return st;
    if (per_sm < 1) per_sm = 1;
    if (dev >= 0 && dev < 64) known[dev].store(per_sm, std::memory_order_release);
  }
  *out = per_sm;
  return CMC_OK;
}

template <int D, int G, bool FUSED, bool PREP>
static int launch_weighted(WeightedParams& p, const cmc_dims& m, cudaStream_t s, int* ctas) {
  int per_sm = 1;
  int st = per_sm_of<D, G, FUSED, PREP>(&per_sm);
  if (st != CMC_OK) return st;
  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  p.cm = plan_cm(m, per_sm);
  if (ctas) {
    *ctas = static_cast<int>(units * p.cm);
    return CMC_OK;
  }
  p.iters = iters_of(m, p.cm);
  size_t bytes = score_bytes(m, p.cm);
  if (bytes > kScoreBytes) bytes = 0;  // in the workspace
  else p.scratch = nullptr;
  p.prefetch = std::min({l2_prefetch_setting(), 3, p.iters});
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.cm);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(units * p.cm));
  cfg.blockDim = dim3(kWThreads);
  cfg.dynamicSmemBytes = WSmem<D, G, PREP>::kScores + bytes;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = p.cm > 1 ? 2 : 1;
  return record_cuda_error(cudaLaunchKernelEx(&cfg, weighted_attn_kernel<D, G, FUSED, PREP>, p));
}

template <bool FUSED, bool PREP>
static int dispatch_weighted(WeightedParams& p, const cmc_dims& m, cudaStream_t s, int* ctas) {
  const int G = m.Hq / m.Hkv;
  if (m.d == 128) {
    switch (G) {
      case 1: return launch_weighted<128, 1, FUSED, PREP>(p, m, s, ctas);
      case 2: return launch_weighted<128, 2, FUSED, PREP>(p, m, s, ctas);
      case 4: return launch_weighted<128, 4, FUSED, PREP>(p, m, s, ctas);
      default: return launch_weighted<128, 8, FUSED, PREP>(p, m, s, ctas);
    }
  }
  switch (G) {
    case 1: return launch_weighted<64, 1, FUSED, PREP>(p, m, s, ctas);
    case 2: return launch_weighted<64, 2, FUSED, PREP>(p, m, s, ctas);
    case 4: return launch_weighted<64, 4, FUSED, PREP>(p, m, s, ctas);
    default: return launch_weighted<64, 8, FUSED, PREP>(p, m, s, ctas);
  }
}

static int check_weighted_dims(const cmc_dims* dims) {
  int st = validate_dims(dims, true);
  if (st != CMC_OK) return st;
  const cmc_dims& m = *dims;
  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  if (units * m.N >= (1LL << 40) || units * m.W >= (1LL << 40)) return CMC_ERR_SHAPE;
  return CMC_OK;
}

static int run_weighted(const void* q, const void* t1k, const void* t1v, float* t1w, void* ring_k,
                        void* ring_v, float* ring_w, int64_t* pos, const void* k_new, const void* v_new,
                        const cmc_dims* dims, float scale, const cmc_qk_prep* prep, void* out,
                        void* workspace, size_t workspace_bytes, void* stream, bool fused) {
  int st = check_weighted_dims(dims);
  if (st != CMC_OK) return st;
  const cmc_dims& m = *dims;
  if (!q || !ring_k || !ring_v || !ring_w || !pos || !out) return CMC_ERR_NULL;
  if (m.k > 0 && (!t1k || !t1v || !t1w)) return CMC_ERR_NULL;
  if (fused && (!k_new || !v_new)) return CMC_ERR_NULL;
  if (!aligned16(q) || !aligned16(t1k) || !aligned16(t1v) || !aligned16(ring_k) || !aligned16(ring_v) ||
      !aligned16(out) || !aligned16(k_new) || !aligned16(v_new) ||
      ((reinterpret_cast<uintptr_t>(t1w) | reinterpret_cast<uintptr_t>(ring_w)) & 3) ||
      (reinterpret_cast<uintptr_t>(pos) & 7))
    return CMC_ERR_ALIGN;
  if (!workspace || workspace_bytes < weighted_ws(m)) return CMC_ERR_WORKSPACE;
  if (!aligned16(workspace)) return CMC_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  WeightedParams p;
  st = prep_params(fused ? prep : nullptr, m.d, s, &p.prep);
  if (st != CMC_OK) return st;
  p.q = static_cast<const uint16_t*>(q);
  p.t1k = static_cast<const uint16_t*>(t1k);
  p.t1v = static_cast<const uint16_t*>(t1v);
  p.t1w = t1w;
  p.ring_k = static_cast<uint16_t*>(ring_k);
  p.ring_v = static_cast<uint16_t*>(ring_v);
  p.ring_w = ring_w;
  p.pos = pos;
  p.k_new = static_cast<const uint16_t*>(k_new);
  p.v_new = static_cast<const uint16_t*>(v_new);
  p.out = static_cast<uint16_t*>(out);
  char* ws = static_cast<char*>(workspace);
  p.status = reinterpret_cast<uint32_t*>(ws);
  p.tickets = reinterpret_cast<unsigned long long*>(ws + kWsHeader);
  p.scratch = reinterpret_cast<float*>(ws + ws_partials_off(m.B));
  p.L = m.L; p.Hkv = m.Hkv; p.N = m.N; p.k = m.k; p.W = m.W; p.LH = m.L * m.Hkv;
  p.cm = 1;
  p.nb1 = (m.k + kBlkKeys - 1) / kBlkKeys;
  const float sc = scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(m.d));
  p.scale_log2 = sc * 1.4426950408889634f;
  if (!fused) return dispatch_weighted<false, false>(p, m, s, nullptr);
  if (p.prep.rope || p.prep.q_weight || p.prep.k_weight) return dispatch_weighted<true, true>(p, m, s, nullptr);
  return dispatch_weighted<true, false>(p, m, s, nullptr);
}

}  // namespace cmc

extern "C" {

size_t cmc_decode_attn_weighted_workspace_size(const cmc_dims* dims) {
  if (cmc::check_weighted_dims(dims) != CMC_OK) return 0;
  return cmc::weighted_ws(*dims);
}

int cmc_decode_attn_weighted_plan(const cmc_dims* dims, int fused, int* ctas) {
  int st = cmc::check_weighted_dims(dims);
  if (st != CMC_OK) return st;
  if (!ctas) return CMC_ERR_NULL;
  cmc::WeightedParams p;
  return fused ? cmc::dispatch_weighted<true, false>(p, *dims, nullptr, ctas)
               : cmc::dispatch_weighted<false, false>(p, *dims, nullptr, ctas);
}

int cmc_two_tier_decode_attn_weighted(const void* q, const void* tier1_k, const void* tier1_v,
                                      float* tier1_weight, const void* ring_k, const void* ring_v,
                                      float* ring_weight, const int64_t* pos, const cmc_dims* dims,
                                      float scale, void* out, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  return cmc::run_weighted(q, tier1_k, tier1_v, tier1_weight, const_cast<void*>(ring_k),
                           const_cast<void*>(ring_v), ring_weight, const_cast<int64_t*>(pos), nullptr,
                           nullptr, dims, scale, nullptr, out, workspace, workspace_bytes, stream, false);
}

int cmc_decode_step_weighted(const void* q, const void* tier1_k, const void* tier1_v, float* tier1_weight,
                             void* ring_k, void* ring_v, float* ring_weight, int64_t* pos,
                             const void* k_new, const void* v_new, const cmc_dims* dims, float scale,
                             const cmc_qk_prep* prep, void* out, void* workspace, size_t workspace_bytes,
                             void* stream) {
  return cmc::run_weighted(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v, ring_weight, pos, k_new,
                           v_new, dims, scale, prep, out, workspace, workspace_bytes, stream, true);
}

}  // extern "C"
